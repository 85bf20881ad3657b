// Dense softmax attention forward in fp32 products, with row statistics, for calls of few queries: tiles of 64 queries, whose
// keys several workgroups may share.
//
// O = softmax(scale Q K^T) V in one pass over the keys: a row keeps a reference m, the sum of 2^(z - m) over its logits z
// (base 2) and the sum of these weights times the values; m is raised only when a logit exceeds it by more than kGrow.
// Layout as in mrt_dense_bwd_f32.hip.  v_mfma_f32_16x16x4_f32 goes at a sixteenth of the bf16 rate, so the kernel of split
// operands (mrt_f32_kernels.hpp, tiles of 128 queries) is ahead by a fifth where its tiles fill the chip; this one where
// they do not (us: 576 tokens of 64 features, one head 39 -> 15, 1560 tokens of 128, 12 heads 246 -> 174).
#include "mrt_dense_train.hpp"
#include "mrt_f32_rows.hpp"

namespace mrt {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 16 * kWaves, kStep = 16;
constexpr float kGrow = 8.0f, kNoKey = -__FLT_MAX__;
template <int D> constexpr int kLd = D + 4;                          // LDS row stride in floats
template <int D> constexpr int kSlot = 2 * kStep * kLd<D>;

__device__ inline f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

template <int D, typename T, bool VEC, bool PART>
__global__ __launch_bounds__(kThreads, 2) void k_f32_dense_fwd(DenseFwd p) {
  constexpr int KS = D / 16, BLK = D / 64, LD = kLd<D>, QUADS = kStep * D / 4 / kThreads;
  __shared__ __attribute__((aligned(16))) float lds[2 * kSlot<D>];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int n_heads = p.B * p.H, d = p.d, tiles = (p.Nq + kRows - 1) / kRows, parts = PART ? p.parts : 1;
  int unit = blockIdx.x;
  const int bh = unit % n_heads;
  unit /= n_heads;
  const int part = unit % parts, tile = tiles - 1 - unit / parts;      // under a mask the longest first
  const int b = bh / p.H, hd = bh - b * p.H, kvh = hd / p.group;
  const int q0 = tile * kRows, keys = dense_keys(p, b), q_last = q0 + kRows < p.Nq ? q0 + kRows - 1 : p.Nq - 1;
  const int k_end = dense_last_key(p, q_last, keys), all = (k_end + kStep - 1) / kStep;
  const int i0 = PART ? (int)((long long)all * part / parts) : 0, i1 = PART ? (int)((long long)all * (part + 1) / parts) : all;
  const T* Kp = (const T*)p.K + b * p.k.batch + kvh * p.k.head;
  const T* Vp = (const T*)p.V + b * p.v.batch + kvh * p.v.head;

  f32x4 rk[QUADS], rv[QUADS];
  auto fetch = [&](int i) {
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
      const int at = tid + j * kThreads, r = kStep * i + at / (D / 4), v = 4 * (at % (D / 4));
      const bool in = r < k_end;
      const long long rr = in ? r : k_end - 1;
      rk[j] = blank4<VEC>(ld4<VEC>(Kp + rr * p.k.token, v, d), v, d);
      rv[j] = blank4<VEC>(ld4<VEC>(Vp + rr * p.v.token, v, d), v, d);
      if (!in) rk[j] = rv[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  auto commit = [&](int slot) {
    float* at = lds + slot * kSlot<D>;
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
      const int q = tid + j * kThreads, r = q / (D / 4), v = 4 * (q % (D / 4));
      *(f32x4*)(at + r * LD + v) = rk[j];
      *(f32x4*)(at + (kStep + r) * LD + v) = rv[j];
    }
  };
  if (i0 < i1) {
    fetch(i0);
    commit(0);
  }
  const int qi = q0 + 16 * wave + c, qc = qi < p.Nq ? qi : p.Nq - 1, lim = dense_last_key(p, qc, keys);
  const T* Qp = (const T*)p.Q + b * p.q.batch + hd * p.q.head + (long long)qc * p.q.token;
  f32x4 qf[KS], o[BLK][4];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = blank4<VEC>(ld4<VEC>(Qp, 16 * ks + 4 * g, d), 16 * ks + 4 * g, d);
#pragma unroll
  for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[blk][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float scale2 = p.scale * kLog2e;
  float m = kNoKey, sum = 0.f;           // reference (the same in the four lanes of a query), this lane's sum

  for (int i = i0; i < i1; ++i) {
    __syncthreads();
    const float* at = lds + ((i - i0) & 1) * kSlot<D>;
    if (i + 1 < i1) fetch(i + 1);
    f32x4 s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const f32x4 a = *(const f32x4*)(at + c * LD + 16 * ks + 4 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = mfma4(a[e], qf[ks][e], s[e]);
    }
    f32x4 w = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int r = 0; r < 4; ++r) w[r] = kStep * i + 4 * g + r < lim ? mul_rounded(w[r], scale2) : -INFINITY;
    const float top = fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3]));
    if (__builtin_amdgcn_ballot_w64(top > m + kGrow) != 0) {           // (also the first logit)
      const float raised = fmaxf(m, xmax(top)), f = exp2_fast(m - raised);
      m = raised;
      sum *= f;
#pragma unroll
      for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[blk][e] = o[blk][e] * f;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      w[r] = exp2_fast(w[r] - m);
      sum += w[r];
    }
    const float* av = at + (kStep + 4 * g) * LD + 4 * c;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int blk = 0; blk < BLK; ++blk) {
        const f32x4 v = *(const f32x4*)(av + r * LD + 64 * blk);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[blk][e] = mfma4(v[e], w[r], o[blk][e]);
      }
    if (i + 1 < i1) commit((i + 1 - i0) & 1);
  }
  sum = xsum(sum);
  if (qi >= p.Nq) return;
  const long long row = (long long)bh * p.Nq + qi, rows = (long long)n_heads * p.Nq;
  const float inv = PART ? 1.f : sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int blk = 0; blk < BLK; ++blk)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int v = 64 * blk + 16 * g + 4 * r;
      const f32x4 x = f32x4{o[blk][0][r], o[blk][1][r], o[blk][2][r], o[blk][3][r]} * inv;
      if constexpr (PART) st4<VEC>(p.po + (part * rows + row) * d, x, v, d);
      else st4<VEC>((T*)p.O + b * p.o.batch + hd * p.o.head + qi * p.o.token, x, v, d);
    }
  if (g == 0) {
    if constexpr (PART) p.ml[part * rows + row] = make_float2(m, sum);
    else p.lse[row] = natural_lse(m, sum);
  }
}

// O and the statistics from the parts, all against the largest reference.  A thread owns four features of a row.
template <typename T, bool VEC>
__global__ __launch_bounds__(kJoinThreads) void k_f32_dense_join(DenseFwd p, long long rows) {
  // (parts have at most 2^27 elements together: 32 bits hold the threads' numbers)
  const int d = p.d;
  const unsigned quads = (d + 3) >> 2, at = blockIdx.x * kJoinThreads + threadIdx.x, row = at / quads;
  const int v = 4 * (int)(at - row * quads);
  if (row >= rows) return;
  constexpr int AHEAD = 8;               // parts in flight: what a thread waits for is memory
  float m = kNoKey, sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < p.parts; i0 += AHEAD) {
    float2 ml[AHEAD];
    f32x4 x[AHEAD];
    float top = m;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const long long from = (i0 + k < p.parts ? i0 + k : p.parts - 1) * rows + row;
      ml[k] = p.ml[from];
      x[k] = ld4<VEC>(p.po + from * d, v, d);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) top = fmaxf(top, ml[k].x);
    const float keep = exp2_fast(m - top);
    m = top;
    sum *= keep;
    o = o * keep;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (i0 + k < p.parts) {
        const float f = exp2_fast(ml[k].x - m);
        sum += ml[k].y * f;
        o = o + x[k] * f;
      }
  }
  const unsigned bh = row / (unsigned)p.Nq, q = row - bh * p.Nq, b = bh / p.H, hd = bh - b * p.H;
  st4<VEC>((T*)p.O + b * p.o.batch + hd * p.o.head + q * p.o.token, o * (sum > 0.f ? 1.f / sum : 0.f), v, d);
  if (v == 0) p.lse[row] = natural_lse(m, sum);
}

template <int D, typename T, bool VEC>
hipError_t run(const DenseFwd& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.Nq + kRows - 1) / kRows * (long long)(p.B * p.H) * p.parts));
  if (p.parts == 1) {
    k_f32_dense_fwd<D, T, VEC, false><<<grid, kThreads, 0, s>>>(p);
    return hipGetLastError();
  }
  k_f32_dense_fwd<D, T, VEC, true><<<grid, kThreads, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long rows = (long long)p.B * p.H * p.Nq;
  k_f32_dense_join<T, VEC><<<(unsigned)((rows * ((p.d + 3) / 4) + kJoinThreads - 1) / kJoinThreads), kJoinThreads, 0, s>>>(p, rows);
  return hipGetLastError();
}
template <typename T>
hipError_t run_t(const DenseFwd& p, hipStream_t s) {
  if (f32_dense_fwd_quads(p, sizeof(T))) return p.d <= 64 ? run<64, T, true>(p, s) : run<128, T, true>(p, s);
  return p.d <= 64 ? run<64, T, false>(p, s) : run<128, T, false>(p, s);
}

// How many workgroups share the keys of a tile: as many as promise the least time by this model.  A step takes t
// microseconds where a compute unit has one workgroup, 1.5 t where it has two (under a mask a long one and one of mean
// length); a join costs a launch and the parts' bytes.
struct DenseShare {
  int parts;
  double us;
};
DenseShare dense_share(long long rows, int tile, long long heads, int d, double t, double first, double last) {
  const double cus = compute_units(), longest = std::max(first, last), mean = 0.5 * (first + last);
  const long long tiles = (rows + tile - 1) / tile * heads, elements = rows * heads * d;
  auto time = [&](int parts) {
    const double each = tiles * parts / cus, pairs = std::floor(each / 2), rest = each - 2 * pairs;
    const double rounds = 1.5 * pairs + (rest > 1 ? 1.5 : rest > 0 ? 1.0 : 0.0);
    const double alone = std::ceil(longest / parts), beside = rounds < 1.5 ? alone : 0.75 * (alone + std::ceil(mean / parts));
    const double steps = std::max(beside, rounds > 1.5 ? (mean / parts + 1) * rounds : 0.0);
    return steps * t + (parts > 1 ? 4.0 + 1.3e-6 * elements * parts : 0.0);
  };
  int best = 1;
  double least = time(1) * 0.95;      // (sharing has to promise 5 %)
  for (int parts = 2; parts <= kMostParts && 2 * parts <= longest && elements * parts <= kMostPartElements; ++parts) {
    const double us = time(parts);
    if (us < least) { least = us; best = parts; }
  }
  return {best, time(best)};
}

}  // namespace

bool f32_dense_fwd_quads(const DenseFwd& p, size_t bytes) {
  const void* ptrs[4] = {p.Q, p.K, p.V, p.O};
  const mrt_strides* st[4] = {&p.q, &p.k, &p.v, &p.o};
  bool quads = p.d % 4 == 0;
  for (int i = 0; i < 4; ++i)
    quads = quads && (uintptr_t)ptrs[i] % (4 * bytes) == 0 && st[i]->token % 4 == 0 && st[i]->head % 4 == 0 && st[i]->batch % 4 == 0;
  return quads;
}

// The other kernel takes 32 keys in 5.0 us at 128 features and 2.1 at 64 (one workgroup of 128 queries to a compute unit;
// two share it at 1.35 times that), and a step of its own, of which a quarter is hidden, for every chunk of a mask that ends
// inside its queries.  This one takes a fifth longer than dense_share says where it fills the chip.  (us, this kernel | the
// other: 16 heads of 1800 tokens 284 | 270, 12 of 5400 tokens of 64 features in chunks of 1800 595 | 429, 16 of 4096 causal
// tokens 688 | 1290, 4 of 600 24 | 82.)
int f32_dense_fwd_parts(const DenseFwd& p) {
  const double first = dense_last_key(p, std::min(kRows, p.Nq) - 1, p.Nkv), last = dense_last_key(p, p.Nq - 1, p.Nkv), cus = compute_units();
  const DenseShare own = dense_share(p.Nq, kRows, (long long)p.B * p.H, p.d, p.d <= 64 ? 0.75 : 1.4, first / kStep, last / kStep);
  const double ends = p.cc > 0 && first != last ? 24.0 * std::max(0.0, 128.0 / ((double)p.cc * p.hw) - 1) : 0.0;
  const double each = (p.Nq + 127) / 128 * (double)(p.B * p.H) / cus, pairs = std::floor(each / 2), rest = each - 2 * pairs;
  const double rounds = first == last ? 1.35 * pairs + (rest > 1 ? 1.35 : rest > 0 ? 1.0 : 0.0) : each <= 1 ? 1.0 : std::max(1.35, 0.675 * each + 0.35);
  const double other = (p.d <= 64 ? 2.1 : 5.0) / 32 * std::max((last + ends) * std::min(rounds, 1.35), (0.5 * (first + last) + ends) * rounds);
  return 1.2 * own.us < other ? own.parts : 0;
}

hipError_t launch_f32_dense_fwd(const DenseFwd& p, int dtype, hipStream_t s) {
  return dtype == MRT_F32 ? run_t<float>(p, s) : run_t<u16>(p, s);
}

}  // namespace mrt
