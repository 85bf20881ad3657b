// Backward pass of the dense softmax attention in fp32 arithmetic, and the sums of its parts.
//
// Products of fp32 operands (v_mfma_f32_16x16x4_f32).  A wave owns 16 rows of one (batch, head), keys (KV) or
// queries, on the N side: their operands and gradients stay in its registers, and the rows of the other side
// stream through LDS, 16 a step.  With feature 16 ks + 4 g + e as slot g of step (ks, e) a lane's operands of
// four steps are 16 contiguous bytes; register r of a logit tile (streamed rows 4 g + r) is as it stands the
// second products' operand of step r.  Those take 16 bytes of a row for four result tiles: lane c reads the
// features 64 blk + 4 c + e of tile e, so register r of the four tiles is feature 64 blk + 16 g + 4 r + e.
#include "mrt_dense_train.hpp"
#include "mrt_f32_rows.hpp"


namespace mrt {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 16 * kWaves, kStep = 16;
template <int D> constexpr int kLd = D + 4;                          // LDS row stride in floats
template <int D> constexpr int kSlot = 2 * kStep * kLd<D> + 2 * kStep;

__device__ inline f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

typedef __attribute__((ext_vector_type(16))) float f32x16;
__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
// features v .. v + 7 of a row as they are stored, zeros from d on (EIGHT: in one access, rows of whole eights)
template <bool VEC, bool EIGHT>
__device__ inline bf16x8 ld8(const u16* row, int v, int d) {
  if constexpr (EIGHT) {
    typedef __attribute__((ext_vector_type(8), aligned(8))) __bf16 eight;
    const eight x = *(const eight*)(row + (v < d ? v : 0));
    return v < d ? (bf16x8)x : bf16x8{};
  }
  uint2 x[2];
#pragma unroll
  for (int h = 0; h < 2; ++h, v += 4) {
    if constexpr (VEC) {
      x[h] = *(const uint2*)(row + (v < d ? v : 0));
      if (v >= d) x[h] = make_uint2(0, 0);
    } else {
      unsigned y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = row[v + e < d ? v + e : 0];
        if (v + e >= d) y[e] = 0;
      }
      x[h] = make_uint2(y[0] | y[1] << 16, y[2] | y[3] << 16);
    }
  }
  return __builtin_bit_cast(bf16x8, x);
}

template <int D, typename T, bool VEC, bool KV, bool PART>
__device__ __forceinline__ void bwd_tile(const DenseBwd& p, int unit, float* lds) {
  constexpr int KS = D / 16, BLK = D / 64, LD = kLd<D>, QUADS = kStep * D / 4 / kThreads;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int n_own = KV ? p.Nkv : p.Nq, n_heads = p.B * (KV ? p.KH : p.H), d = p.d;
  const int tiles = (n_own + kRows - 1) / kRows, parts = PART ? (KV ? p.parts_kv : p.parts_q) : 1;
  const int bh = unit % n_heads;
  unit /= n_heads;
  const int part = unit % parts, tile = KV ? unit / parts : tiles - 1 - unit / parts;    // under a mask the longest first
  const int b = bh / (KV ? p.KH : p.H), hd = bh - b * (KV ? p.KH : p.H), kvh = KV ? hd : hd / p.group;
  const int own0 = tile * kRows, keys = dense_seen_keys(p, b), own_last = own0 + kRows < n_own ? own0 + kRows - 1 : n_own - 1;

  // the streamed rows: queries qfirst .. Nq of every head that shares these keys, or keys 0 .. last
  const int qfirst = KV ? dense_first_query(p, own0) & ~(kStep - 1) : 0;
  const int s_end = KV ? p.Nq : dense_last_key(p, own_last, keys);
  const int per_head = !KV || own0 < keys ? (s_end - qfirst + kStep - 1) / kStep : 0;
  const int all = KV ? per_head * p.group : per_head;
  const int i0 = PART ? (int)((long long)all * part / parts) : 0, i1 = PART ? (int)((long long)all * (part + 1) / parts) : all;
  const int nqb = (p.Nq + 31) >> 5;

  const T* own_a = KV ? (const T*)p.K + b * p.k.batch + hd * p.k.head : (const T*)p.Q + b * p.q.batch + hd * p.q.head;
  const T* own_b = KV ? (const T*)p.V + b * p.v.batch + hd * p.v.head : (const T*)p.dO + b * p.dout.batch + hd * p.dout.head;
  const long long own_at = KV ? p.k.token : p.q.token, own_bt = KV ? p.v.token : p.dout.token;
  const T* st_a = KV ? (const T*)p.Q + b * p.q.batch + (long long)hd * p.group * p.q.head
                     : (const T*)p.K + b * p.k.batch + kvh * p.k.head;
  const T* st_b = KV ? (const T*)p.dO + b * p.dout.batch + (long long)hd * p.group * p.dout.head
                     : (const T*)p.V + b * p.v.batch + kvh * p.v.head;
  const long long st_at = KV ? p.q.token : p.k.token, st_bt = KV ? p.dout.token : p.v.token;

  f32x4 ra[QUADS], rb[QUADS];
  float rst = 0.f;
  auto fetch = [&](int i) {
    const int gh = KV ? i / per_head : 0, row = KV ? qfirst + kStep * (i - gh * per_head) : kStep * i;
    const T* a = st_a + (KV ? gh * p.q.head : 0);
    const T* bb = st_b + (KV ? gh * p.dout.head : 0);
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
      const int at = tid + j * kThreads, r = row + at / (D / 4), v = 4 * (at % (D / 4));
      const bool in = r < s_end;
      const long long rr = in ? r : s_end - 1;
      ra[j] = blank4<VEC>(ld4<VEC>(a + rr * st_at, v, d), v, d);
      rb[j] = blank4<VEC>(ld4<VEC>(bb + rr * st_bt, v, d), v, d);
      if (!in) ra[j] = rb[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if constexpr (KV)
      if (tid < 2 * kStep) {
        const int r = row + (tid & (kStep - 1));
        rst = p.stats[((long long)(b * p.H + hd * p.group + gh) * nqb + (r >> 5)) * 64 + 32 * (tid / kStep) + (r & 31)];
      }
  };
  auto commit = [&](int slot) {
    float* at = lds + slot * kSlot<D>;
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
      const int q = tid + j * kThreads, r = q / (D / 4), v = 4 * (q % (D / 4));
      *(f32x4*)(at + r * LD + v) = ra[j];
      *(f32x4*)(at + (kStep + r) * LD + v) = rb[j];
    }
    if (KV && tid < 2 * kStep) at[2 * kStep * LD + tid] = rst;
  };
  if (i0 < i1) {
    fetch(i0);
    commit(0);
  }

  const int r_own = own0 + 16 * wave + c, rc = r_own < n_own ? r_own : n_own - 1;
  f32x4 oa[KS], ob[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int v = 16 * ks + 4 * g;
    oa[ks] = blank4<VEC>(ld4<VEC>(own_a + rc * own_at, v, d), v, d);
    ob[ks] = blank4<VEC>(ld4<VEC>(own_b + rc * own_bt, v, d), v, d);
  }
  const int lim = KV ? dense_first_query(p, rc) : dense_last_key(p, rc, keys);
  float nlse = 0.f, ndelta = 0.f;
  if constexpr (!KV) {
    const float* st = p.stats + ((long long)bh * nqb + (rc >> 5)) * 64 + (rc & 31);
    nlse = st[0];
    ndelta = st[32];
  }
  f32x4 g1[BLK][4], g2[BLK][4];
#pragma unroll
  for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
    for (int e = 0; e < 4; ++e) g1[blk][e] = g2[blk][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float scale2 = p.scale * kLog2e;

  for (int i = i0; i < i1; ++i) {
    __syncthreads();
    const float* at = lds + ((i - i0) & 1) * kSlot<D>;
    const float* bt = at + kStep * LD;
    if (i + 1 < i1) fetch(i + 1);
    const int row = KV ? qfirst + kStep * (i % per_head) : kStep * i;
    f32x4 s[4], dp[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = dp[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const f32x4 a = *(const f32x4*)(at + c * LD + 16 * ks + 4 * g), x = *(const f32x4*)(bt + c * LD + 16 * ks + 4 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = mfma4(a[e], oa[ks][e], s[e]);
        dp[e] = mfma4(x[e], ob[ks][e], dp[e]);
      }
    }
    f32x4 w = (s[0] + s[1]) + (s[2] + s[3]), ds = (dp[0] + dp[1]) + (dp[2] + dp[3]);
    f32x4 nl = {nlse, nlse, nlse, nlse}, nd = {ndelta, ndelta, ndelta, ndelta};
    if constexpr (KV) {
      nl = *(const f32x4*)(bt + kStep * LD + 4 * g);
      nd = *(const f32x4*)(bt + kStep * LD + kStep + 4 * g);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int at_row = row + 4 * g + r;
      const bool seen = KV ? at_row >= lim : at_row < lim;
      const float pr = exp2_fast(fmaf(w[r], scale2, nl[r]));
      w[r] = seen ? pr : 0.f;
      ds[r] = seen ? pr * (ds[r] + nd[r]) : 0.f;
    }
    const float* a2 = at + 4 * g * LD + 4 * c;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int blk = 0; blk < BLK; ++blk) {
        const f32x4 y = *(const f32x4*)(a2 + r * LD + 64 * blk);
#pragma unroll
        for (int e = 0; e < 4; ++e) g2[blk][e] = mfma4(y[e], ds[r], g2[blk][e]);
        if constexpr (KV) {
          const f32x4 x = *(const f32x4*)(a2 + (kStep + r) * LD + 64 * blk);
#pragma unroll
          for (int e = 0; e < 4; ++e) g1[blk][e] = mfma4(x[e], w[r], g1[blk][e]);
        }
      }
    if (i + 1 < i1) commit((i + 1 - i0) & 1);
  }
  if (r_own >= n_own) return;
  const bool live = KV ? r_own < keys : true;
#pragma unroll
  for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int v = 64 * blk + 16 * g + 4 * r;
      f32x4 x, y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = live ? p.scale * g2[blk][e][r] : 0.f;
        y[e] = live ? g1[blk][e][r] : 0.f;
      }
      if constexpr (PART) {
        const long long to = (((long long)part * n_heads + bh) * n_own + r_own) * d;
        st4<VEC>((KV ? p.pk : p.pq) + to, x, v, d);
        if (KV) st4<VEC>(p.pv + to, y, v, d);
      } else if constexpr (KV) {
        st4<VEC>((T*)p.dK + b * p.dk.batch + hd * p.dk.head + r_own * p.dk.token, x, v, d);
        st4<VEC>((T*)p.dV + b * p.dv.batch + hd * p.dv.head + r_own * p.dv.token, y, v, d);
      } else {
        st4<VEC>((T*)p.dQ + b * p.dq.batch + hd * p.dq.head + r_own * p.dq.token, x, v, d);
      }
    }
}

// One launch for both: the key tiles, whose steps are the longer ones, come first.
template <int D, typename T, bool VEC, bool PART_Q, bool PART_KV>
__global__ __launch_bounds__(kThreads, 2) void k_f32_dense_bwd(DenseBwd p, int key_units) {
  __shared__ __attribute__((aligned(16))) float lds[2 * kSlot<D>];
  const int unit = blockIdx.x;
  if (unit < key_units) bwd_tile<D, T, VEC, true, PART_KV>(p, unit, lds);
  else bwd_tile<D, T, VEC, false, PART_Q>(p, unit - key_units, lds);
}

// What the tiles need of a row of queries: -log2(e) lse (-infinity where it sees no key: weights of zero) and -delta,
// delta the sum of its O dO.  64 numbers for 32 rows, rows behind the last one as such that see no key.  Sixteen threads a
// row; memory bounds it.
//
// bf16 storage: O was rounded to bf16, and where rows see few keys delta then costs as much as the rounding of the results
// (10 causal tokens of 128 features: dQ and dK 2.3e-3 of the 2-norm off instead of 1.7e-3, 100 of them 1.9e-3 instead of
// 1.7e-3), where their values are alike several times as much.  So 32 rows that all see at most kFewKeys keys form delta as
// the sum of P dP, a tile of 32 keys a wave.  Products of bf16 numbers are exact in 32 bits, so that the bf16 matrix unit
// forms the same sums as the fp32 one.  The loads bound it: whole rows of eights as 16 bytes (64 heads of 100 causal tokens
// of 128 features, us of the launch: 9.6, in eights of 8 bytes 15.3; with fp32 products, sixteen rows a workgroup, the
// heads one by one 16.1; 3.3 with dO . O).
constexpr int kFewKeys = 32 * kWaves;
template <int D, typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void k_f32_dense_bwd_stats(DenseBwd p, int nqb) {
  // (heads in turn: where there are eight or more, the workgroups of one reach the same XCD, whose L2 has its keys)
  const unsigned heads = p.B * p.H, block = blockIdx.x / heads;
  const int bh = blockIdx.x - block * heads, r0 = 16 * (block & 1), q0 = (int)(block >> 1) * 32;
  const int b = bh / p.H, hd = bh - b * p.H;
  float* st = p.stats + ((long long)bh * nqb + (block >> 1)) * 64;
  const T* Op = (const T*)p.O + b * p.o.batch + hd * p.o.head;
  const T* dOp = (const T*)p.dO + b * p.dout.batch + hd * p.dout.head;
  auto negative_lse = [&](int q) {
    const float lse = q < p.Nq ? p.lse[(long long)bh * p.Nq + q] : -INFINITY;
    return lse == -INFINITY ? -INFINITY : -kLog2e * lse;
  };
  if constexpr (sizeof(T) == 2) {
    const int keys = dense_seen_keys(p, b), most = dense_last_key(p, q0 + 31 < p.Nq ? q0 + 31 : p.Nq - 1, keys);
    if (most > 0 && most <= kFewKeys) {
      if (r0 > 0) return;                // (all rows are the other workgroup's)
      constexpr int KS = D / 16;
      __shared__ float sums[kWaves][32];
      const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, hi = lane >> 5, c = lane & 31;
      const int q = q0 + c, k0 = 32 * wave, lim = q < p.Nq ? dense_last_key(p, q, keys) : 0;
      const long long qr = q < p.Nq ? q : p.Nq - 1, kr = k0 + c < most ? k0 + c : most - 1;
      const T* Qr = (const T*)p.Q + b * p.q.batch + hd * p.q.head + qr * p.q.token;
      const T* Gr = dOp + qr * p.dout.token;
      const T* Kr = (const T*)p.K + b * p.k.batch + hd / p.group * p.k.head + kr * p.k.token;
      const T* Vr = (const T*)p.V + b * p.v.batch + hd / p.group * p.v.head + kr * p.v.token;
      const float nl = negative_lse(q), scale2 = p.scale * kLog2e;
      f32x16 s = {}, dp = {};            // rows: keys k0 + 8 (r >> 2) + 4 hi + (r & 3); columns: queries
      auto products = [&](auto eight) {
        constexpr bool E = VEC && decltype(eight)::value;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int v = 16 * ks + 8 * hi;
          s = mfma32(ld8<VEC, E>(Kr, v, p.d), ld8<VEC, E>(Qr, v, p.d), s);
          dp = mfma32(ld8<VEC, E>(Vr, v, p.d), ld8<VEC, E>(Gr, v, p.d), dp);
        }
      };
      if (p.d % 8 == 0) products(std::true_type{});
      else products(std::false_type{});
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = exp2_fast(fmaf(s[r], scale2, nl)) * dp[r];
        sum += k0 + 8 * (r >> 2) + 4 * hi + (r & 3) < lim ? x : 0.f;
      }
      sum += __shfl_xor(sum, 32);
      if (hi == 0) sums[wave][c] = sum;
      __syncthreads();
      if (tid < 32) {
        st[c] = nl;
        st[32 + c] = -((sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]));
      }
      return;
    }
  }
  const int r = r0 + (threadIdx.x >> 4), q = q0 + r, row = q < p.Nq ? q : p.Nq - 1;
  const T *o = Op + row * p.o.token, *dO = dOp + row * p.dout.token;
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int v = 4 * (threadIdx.x & 15) + 64 * k;
    const f32x4 x = blank4<VEC>(ld4<VEC>(o, v, p.d), v, p.d), y = blank4<VEC>(ld4<VEC>(dO, v, p.d), v, p.d);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum = fmaf(x[e], y[e], sum);
  }
#pragma unroll
  for (int m = 8; m > 0; m >>= 1) sum += __shfl_xor(sum, m, 16);
  if ((threadIdx.x & 15) == 0) {
    st[r] = negative_lse(q);
    st[32 + r] = q >= p.Nq ? 0.f : -sum;
  }
}

// Gradients from their parts, added in their order: those of dQ, dK and dV that have some (blockIdx.y).  A thread owns four features of a
// row and has two or eight parts in flight: what it waits for is memory.
struct JoinArgs {
  struct {
    const float* from;
    void* to;
    mrt_strides st;
    long long rows;
    int n, tokens, heads;
  } a[3];
};
// (parts have at most 2^27 elements together: 32 bits hold the threads' numbers)
template <typename T, bool VEC, int AHEAD>
__global__ __launch_bounds__(kJoinThreads) void k_dense_bwd_join(JoinArgs args, int d) {
  const auto& a = args.a[blockIdx.y];
  const int n = a.n;
  const unsigned quads = (d + 3) >> 2, at = blockIdx.x * kJoinThreads + threadIdx.x, row = at / quads;
  const int v = 4 * (int)(at - row * quads);
  if (row >= a.rows) return;
  const float* from = a.from + (long long)row * d;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < n; i += AHEAD) {
    f32x4 y[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) y[k] = ld4<VEC>(from + (i + k < n ? i + k : n - 1) * a.rows * d, v, d);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (i + k < n) x = x + y[k];
  }
  const unsigned bh = row / (unsigned)a.tokens, tok = row - bh * a.tokens, b = bh / a.heads, hd = bh - b * a.heads;
  st4<VEC>((T*)a.to + b * a.st.batch + hd * a.st.head + tok * a.st.token, x, v, d);
}
template <typename T, bool VEC>
void join(const JoinArgs& a, int most, dim3 grid, int d, hipStream_t s) {
  if (most <= 2) k_dense_bwd_join<T, VEC, 2><<<grid, kJoinThreads, 0, s>>>(a, d);
  else k_dense_bwd_join<T, VEC, 8><<<grid, kJoinThreads, 0, s>>>(a, d);
}

template <int D, typename T, bool VEC>
hipError_t run_both(const DenseBwd& p, int dtype, hipStream_t s) {
  const int nqb = (p.Nq + 31) / 32;
  k_f32_dense_bwd_stats<D, T, VEC><<<2 * (unsigned)(p.B * p.H) * nqb, kThreads, 0, s>>>(p, nqb);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long keys = (p.Nkv + kRows - 1) / kRows * (long long)(p.B * p.KH) * p.parts_kv;
  const long long queries = (p.Nq + kRows - 1) / kRows * (long long)(p.B * p.H) * p.parts_q;
  const bool pq = p.parts_q > 1, pkv = p.parts_kv > 1;
  const auto kernel = pq ? pkv ? k_f32_dense_bwd<D, T, VEC, true, true> : k_f32_dense_bwd<D, T, VEC, true, false>
                         : pkv ? k_f32_dense_bwd<D, T, VEC, false, true> : k_f32_dense_bwd<D, T, VEC, false, false>;
  kernel<<<(unsigned)(keys + queries), kThreads, 0, s>>>(p, (int)keys);
  e = hipGetLastError();
  return e != hipSuccess || !(pq || pkv) ? e : launch_dense_bwd_join(p, pq, pkv, dtype, s);
}
template <typename T>
bool rows_of_four(const DenseBwd& p) {
  const void* ptrs[8] = {p.Q, p.K, p.V, p.O, p.dO, p.dQ, p.dK, p.dV};
  const mrt_strides* st[8] = {&p.q, &p.k, &p.v, &p.o, &p.dout, &p.dq, &p.dk, &p.dv};
  if (p.d % 4) return false;
  for (int i = 0; i < 8; ++i)
    if ((uintptr_t)ptrs[i] % (4 * sizeof(T)) || st[i]->token % 4 || st[i]->head % 4 || st[i]->batch % 4) return false;
  return true;
}
template <typename T>
hipError_t run_t(const DenseBwd& p, int dtype, hipStream_t s) {
  if (rows_of_four<T>(p)) return p.d <= 64 ? run_both<64, T, true>(p, dtype, s) : run_both<128, T, true>(p, dtype, s);
  return p.d <= 64 ? run_both<64, T, false>(p, dtype, s) : run_both<128, T, false>(p, dtype, s);
}

}  // namespace

hipError_t launch_dense_bwd_join(const DenseBwd& p, bool q, bool kv, int dtype, hipStream_t s) {
  const long long rq = (long long)p.B * p.H * p.Nq, rkv = (long long)p.B * p.KH * p.Nkv;
  JoinArgs a;
  int n = 0;
  if (q) a.a[n++] = {p.pq, p.dQ, p.dq, rq, p.parts_q, p.Nq, p.H};
  if (kv) {
    a.a[n++] = {p.pk, p.dK, p.dk, rkv, p.parts_kv, p.Nkv, p.KH};
    a.a[n++] = {p.pv, p.dV, p.dv, rkv, p.parts_kv, p.Nkv, p.KH};
  }
  const long long threads = (q && kv ? std::max(rq, rkv) : q ? rq : rkv) * ((p.d + 3) / 4);
  const dim3 grid((unsigned)((threads + kJoinThreads - 1) / kJoinThreads), n);
  const int most = std::max(q ? p.parts_q : 0, kv ? p.parts_kv : 0);
  const bool bf16 = dtype == MRT_BF16, vec = bf16 ? rows_of_four<u16>(p) : rows_of_four<float>(p);
  if (bf16 && vec) join<u16, true>(a, most, grid, p.d, s);
  else if (bf16) join<u16, false>(a, most, grid, p.d, s);
  else if (vec) join<float, true>(a, most, grid, p.d, s);
  else join<float, false>(a, most, grid, p.d, s);
  return hipGetLastError();
}

// (us without sharing, shared in two launches, and in one: one head of 576 tokens of 64 features 109 | 34 | 25, 12 heads of
// 1560 tokens of 128 790 | 593 | 550)
DenseBwdShape f32_dense_bwd_shape(const DenseBwd& p) {
  return dense_bwd_shape(p, kRows, kStep, p.d <= 64 ? 0.95 : 1.84, p.d <= 64 ? 1.33 : 2.73);
}

hipError_t launch_f32_dense_bwd(const DenseBwd& p, int dtype, hipStream_t s) {
  return dtype == MRT_F32 ? run_t<float>(p, dtype, s) : run_t<u16>(p, dtype, s);
}

}  // namespace mrt
