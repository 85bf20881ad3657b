// Root-mean-square norms of queries and keys, a row of every head by itself, with rotary positions in the same pass.
//
//   r = 1 / sqrt(mean(x x) + eps)     y = turn(r x w)
//   g = turn back(dy)   n = r x   dx = r (g w - n mean(g w n))   dw = sum over rows of g n
//
// Every element is read and written once: memory bounds the call (12 heads of 4680 tokens, Q and K, bf16, 57.5 MB, 12.7 us; gradients of
// 40 heads of 75600, 4.6 GB, 947 us).  A group of lanes, a power of two, owns the rows of a
// token: a lane the same features in every head, so that its angles, which all heads share, are formed once (in
// quarter turns and 64 bits), and its weights and their gradients stay in registers.  Sums over a row are exchanges
// between the lanes of its group.  Gradients of weights: a lane's sums over its rows, joined in LDS for a workgroup and by a
// second launch for the tensor, always in the same order.
#include "mrt_norm_rotary.hpp"
#include "mrt_rotary_rows.hpp"
#include "mrt_bf16_tiles.hpp"

#include <algorithm>

namespace mrt {

namespace {

constexpr int kThreadsNorm = 256;

struct NormTensor {
  const void *x, *dy;
  void* out;
  const void* weight;
  float* parts;                 // of the weights' gradients: [head or 1][part][head_dim]
  float* dweight;
  const int* positions;
  long long pos_batch, pos_axis, weight_head;
  mrt_strides xs, dys, os;
  int heads, tokens, rows;      // rows: batch x tokens
  int h, w, frame0;
  int weight_f32;
  int blocks, runs;             // workgroups along the rows, along the heads
};
struct NormArgs {
  NormTensor t[2];
  double quarters[kMostPairs];  // quarter turns of a pair, per position; negative for the inverse
  int end0, end1, pairs;
  int items, turned, d;
  int lanes;                    // of a row
  int split_block, heads_a_thread, adjacent;
  float eps, inv_d;
};

// Cosine and sine of an angle in quarter turns: the nearest quarter is taken off in 64 bits, which leaves half a quarter at
// most for the Taylor series (the first terms left out are 1.8e-9 and 1.2e-10), and exchanges or negates them.  (Against
// sincospif, which has to take any argument, gradients of 12 heads of 4680 tokens with a weight for every head 32.0 -> 30.9 us.)
__device__ inline void cos_sin(double quarters, float& cs, float& sn) {
  const double whole = rint(quarters);
  const float x = (float)(quarters - whole), y = x * x;
  const int q = (int)whole;
  const float s = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.604411848e-04f, -4.681754135e-03f), 7.969262625e-02f), -6.459640975e-01f), 1.570796327e+00f);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.520204237e-05f, 9.192602748e-04f), -2.086348076e-02f), 2.536695079e-01f), -1.233700550e+00f), 1.0f);
  const float a = q & 1 ? c : s, b = q & 1 ? s : c;
  sn = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, a) ^ ((unsigned)(q & 2) << 30));
  cs = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, b) ^ ((unsigned)((q + 1) & 2) << 30));
}

// The sums of the rows of a batch over their groups of lanes.
template <int N>
__device__ inline void group_sums(float (&x)[N], int lanes) {
  auto each = [&](auto step) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] += step(x[k]);
  };
  if (lanes > 1) each([](float y) { return dpp_mov<0xB1>(y); });
  if (lanes > 2) each([](float y) { return dpp_mov<0x4E>(y); });
  if (lanes > 4) each([](float y) { return dpp_mov<0x141>(y); });
  if (lanes > 8) each([](float y) { return dpp_mov<0x140>(y); });
  if (lanes > 16) each([](float y) { return __shfl_xor(y, 16); });
  if (lanes > 32) each([](float y) { return __shfl_xor(y, 32); });
}

// The accesses of an item, and its numbers: apart, so that all loads of a batch are under way before the first is waited for.
template <typename T, int V, bool HALVES>
struct Raw {
  typename Run<T, V>::type v[HALVES ? 2 : 1];
  __device__ inline void load(const T* at, int f0, int f1) {
    v[0] = *(const typename Run<T, V>::type*)(at + f0);
    if constexpr (HALVES) v[1] = *(const typename Run<T, V>::type*)(at + f1);
  }
  __device__ inline float operator[](int e) const {
    if constexpr (V == 1) return (float)v[e];
    else return (float)v[e / V][e % V];
  }
};

// V, HALVES: elements of an access, as in k_rotary.  ITEMS: of a lane.  AHEAD: heads of a batch, of which one is loaded while
// another is formed (forward two: three and four measured up to 5 % behind; backward two, or one where a lane has one head).
template <typename TX, typename TY, int V, bool HALVES, int ITEMS, bool BWD, int AHEAD>
__global__ __launch_bounds__(kThreadsNorm) void k_norm_rotary(const NormArgs a) {
  constexpr int NP = HALVES ? V : V / 2, N = HALVES ? 2 * V : V;
  typedef typename std::conditional<BWD, TX, TY>::type TO;
  const bool second = (int)blockIdx.x >= a.split_block;
  const NormTensor& t = a.t[second];
  const int block = blockIdx.x - (second ? a.split_block : 0);
  const int h0 = blockIdx.y * a.heads_a_thread, h1 = h0 + a.heads_a_thread < t.heads ? h0 + a.heads_a_thread : t.heads;
  if (h0 >= h1) return;
  const int lane = threadIdx.x & (a.lanes - 1), local = threadIdx.x / a.lanes, rows_a_block = kThreadsNorm / a.lanes;
  const bool next = V == 1 && a.adjacent;
  // a lane's items: pairs to turn, features to copy, or none
  bool there[ITEMS], turns[ITEMS];
  int f0[ITEMS], f1[ITEMS];
  float w[ITEMS][N], dw[ITEMS][N];
  auto weights = [&](int h) {
    if (!t.weight) return;
    const long long row = h * t.weight_head;
    auto read = [&](auto* at) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) w[i][e] = (float)at[row + (e < V ? f0[i] + e : f1[i] + e - V)];
    };
    if (t.weight_f32) read((const float*)t.weight);
    else read((const __bf16*)t.weight);
  };
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int item = lane + i * a.lanes;
    there[i] = item < a.items;
    turns[i] = item < a.turned;
    f0[i] = !turns[i] ? 2 * a.pairs + V * (item - a.turned) : next ? 2 * item : V * item;
    f1[i] = !turns[i] ? f0[i] : next ? f0[i] + 1 : f0[i] + a.pairs;
    if (!there[i]) f0[i] = f1[i] = 0;                // (loads are not conditional, what they bring there is dropped)
#pragma unroll
    for (int e = 0; e < N; ++e) { w[i][e] = 1.f; dw[i][e] = 0.f; }
  }
  const bool whole = a.items == a.lanes * ITEMS && a.turned == a.items;
  // (what does not depend on rows is loaded behind the first row, not before it)
  double quarters[ITEMS][NP];
  bool begun = false;
  for (long long row_l = (long long)block * rows_a_block + local; row_l < t.rows; row_l += (long long)t.blocks * rows_a_block) {
    const int row = (int)row_l, b = row / t.tokens, token = row - b * t.tokens;
    const TX* x = (const TX*)t.x + b * t.xs.batch + token * t.xs.token;
    const TY* dy = (const TY*)t.dy + b * t.dys.batch + token * t.dys.token;
    TO* out = (TO*)t.out + b * t.os.batch + token * t.os.token;
    Raw<TX, V, HALVES> rx[AHEAD][ITEMS];
    Raw<TY, V, HALVES> ry[BWD ? AHEAD : 1][ITEMS];
    auto fetch = [&](int h) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int hk = h + k < h1 ? h + k : h;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          rx[k][i].load(x + hk * t.xs.head, f0[i], f1[i]);
          if constexpr (BWD) ry[k][i].load(dy + hk * t.dys.head, f0[i], f1[i]);
        }
      }
    };
    fetch(h0);
    if (!begun) {
      if (t.weight_head == 0) weights(0);
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < NP; ++e) quarters[i][e] = turns[i] ? a.quarters[(HALVES ? V * (lane + i * a.lanes) : f0[i] / 2) + e] : 0.0;
      begun = true;
    }
    int pos[3];
    if (t.positions) {
      const int* at = t.positions + b * t.pos_batch + token;
#pragma unroll
      for (int axis = 0; axis < 3; ++axis) pos[axis] = at[axis * t.pos_axis];
    } else {
      const int line = token / t.w;
      pos[2] = token - line * t.w;
      const int frame = line / t.h;
      pos[1] = line - frame * t.h;
      pos[0] = frame + t.frame0;
    }
    float cs[ITEMS][NP], sn[ITEMS][NP];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        const int p = (HALVES ? V * (lane + i * a.lanes) : f0[i] / 2) + e, at = p < a.end0 ? pos[0] : p < a.end1 ? pos[1] : pos[2];
        cos_sin(at * quarters[i][e], cs[i][e], sn[i][e]);          // (copied features: 0 turns)
      }
    auto store = [&](TO* at, int i, const float (&v)[N]) {
      if (!there[i]) return;
      float u[V];
#pragma unroll
      for (int e = 0; e < V; ++e) u[e] = v[e];
      store_run(at + f0[i], u);
      if constexpr (HALVES)
        if (turns[i]) {
#pragma unroll
          for (int e = 0; e < V; ++e) u[e] = v[V + e];
          store_run(at + f1[i], u);
        }
    };
    auto turn = [&](int i, float (&v)[N]) {
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        const int p = HALVES ? e : 2 * e, q = HALVES ? V + e : 2 * e + 1;
        const float x0 = v[p], x1 = v[q];
        v[p] = fmaf(x0, cs[i][e], -(x1 * sn[i][e]));
        v[q] = fmaf(x0, sn[i][e], x1 * cs[i][e]);
      }
    };
    for (int h = h0; h < h1; h += AHEAD) {
      // the next batch is under way while this one is formed
      Raw<TX, V, HALVES> was[AHEAD][ITEMS];
      Raw<TY, V, HALVES> gave[BWD ? AHEAD : 1][ITEMS];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          was[k][i] = rx[k][i];
          if constexpr (BWD) gave[k][i] = ry[k][i];
        }
      if (h + AHEAD < h1) fetch(h + AHEAD);
      auto number = [&](const auto& raw, int i, int e) { return whole || (e < V ? there[i] : turns[i]) ? raw[e] : 0.f; };
      float r[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        r[k] = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
          for (int e = 0; e < N; ++e) r[k] = fmaf(number(was[k][i], i, e), number(was[k][i], i, e), r[k]);
      }
      group_sums(r, a.lanes);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) r[k] = rsqrtf(fmaf(r[k], a.inv_d, a.eps));
      if constexpr (!BWD) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          if (h + k >= h1) break;
          if (t.weight_head != 0) weights(h + k);
#pragma unroll
          for (int i = 0; i < ITEMS; ++i) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = number(was[k][i], i, e) * (r[k] * w[i][e]);
            turn(i, v);
            store(out + (h + k) * t.os.head, i, v);
          }
        }
      } else {
        float g[AHEAD][ITEMS][N], along[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          along[k] = 0.f;
          if (t.weight_head != 0) weights(h + k < h1 ? h + k : h);
#pragma unroll
          for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
            for (int e = 0; e < N; ++e) g[k][i][e] = number(gave[k][i], i, e);
            turn(i, g[k][i]);
#pragma unroll
            for (int e = 0; e < N; ++e) {
              const float n = number(was[k][i], i, e) * r[k];
              if (k == 0 || h + k < h1) dw[i][e] = fmaf(g[k][i][e], n, dw[i][e]);
              g[k][i][e] *= w[i][e];
              along[k] = fmaf(g[k][i][e], n, along[k]);
            }
          }
        }
        group_sums(along, a.lanes);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          if (h + k >= h1) break;
          const float by = along[k] * a.inv_d;
#pragma unroll
          for (int i = 0; i < ITEMS; ++i) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = r[k] * fmaf(-by, number(was[k][i], i, e) * r[k], g[k][i][e]);
            store(out + (h + k) * t.os.head, i, v);
          }
        }
      }
    }
  }
  if constexpr (BWD) {
    if (!t.dweight) return;
    // [rows of the workgroup][features]: kThreadsNorm x ITEMS x N numbers at most
    extern __shared__ float sums[];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (there[i])
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e < V || turns[i]) sums[local * a.d + (e < V ? f0[i] + e : f1[i] + e - V)] = dw[i][e];
    __syncthreads();
    // (a head of its own weights: one run, blockIdx.y, a head)
    float* part = t.parts + ((long long)blockIdx.y * t.blocks + block) * a.d;
    for (int f = threadIdx.x; f < a.d; f += kThreadsNorm) {
      float sum = 0.f;
      for (int i = 0; i < rows_a_block; ++i) sum += sums[i * a.d + f];
      part[f] = sum;
    }
  }
}

// The gradients of weights from their parts, in 64 bits: 16 features and 16 runs of parts a workgroup.
struct NormJoin {
  const float* parts[2];
  float* dweight[2];
  int n[2], heads[2];           // parts of a head, heads
  int d;
};
__global__ __launch_bounds__(256) void k_norm_join(const NormJoin j) {
  __shared__ double sums[16][17];
  const int side = blockIdx.z, head = blockIdx.y, n = j.n[side];
  if (head >= j.heads[side]) return;
  const int f = 16 * blockIdx.x + (threadIdx.x & 15), run = threadIdx.x >> 4;
  const float* at = j.parts[side] + (long long)head * n * j.d + (f < j.d ? f : 0);
  double sum = 0;
  for (int i0 = run; i0 < n; i0 += 16 * 8) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = at[(long long)(i0 + 16 * e < n ? i0 + 16 * e : 0) * j.d];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += i0 + 16 * e < n ? x[e] : 0.f;
  }
  sums[run][threadIdx.x & 15] = sum;
  __syncthreads();
  if (threadIdx.x < 16 && f < j.d) {
    sum = 0;
    for (int i = 0; i < 16; ++i) sum += sums[i][threadIdx.x];
    j.dweight[side][(long long)head * j.d + f] = (float)sum;
  }
}

int run_length(const mrt_rotary& r, const mrt_norm_tensor& x, const void* X, const void* dY, const void* out, bool backward, int pairs) {
  const mrt_rotary_tensor& t = x.t;
  const size_t xb = t.x_dtype == MRT_F32 ? 4 : 2, yb = t.y_dtype == MRT_F32 ? 4 : 2;
  const struct { const void* at; const mrt_strides* st; size_t size; } all[3] = {
      {X, &t.x, xb}, {backward ? dY : out, &t.y, yb}, {out, backward ? &x.dx : &t.y, backward ? xb : yb}};
  // (8 elements of both halves, or 8 of 32 bits on both sides, hold more registers than their wider accesses gain: 12 heads of
  // 4680 tokens in halves forward 16.0 -> 13.4 us, backward 37.0 -> 23.6; 9 frames of 1560 in fp32 73 -> 68.)
  for (int v = r.layout == MRT_ROTARY_HALVES || (xb == 4 && yb == 4) ? 4 : 8; v > 1; v /= 2) {
    bool ok = r.head_dim % v == 0 && (r.layout == MRT_ROTARY_ADJACENT ? 2 * pairs : pairs) % v == 0;
    for (const auto& k : all) {
      const size_t bytes = std::min<size_t>(v * k.size, 16);
      ok = ok && (uintptr_t)k.at % bytes == 0 && k.st->token * k.size % bytes == 0 && k.st->head * k.size % bytes == 0 &&
           k.st->batch * k.size % bytes == 0;
    }
    if (ok) return v;
  }
  return 1;
}

template <typename TX, typename TY, bool BWD, int AHEAD>
void run_form(const NormArgs& a, int v, bool halves, dim3 grid, size_t lds, hipStream_t s) {
  if (v == 1) k_norm_rotary<TX, TY, 1, true, 4, BWD, AHEAD><<<grid, kThreadsNorm, lds, s>>>(a);
  else if (halves) {
    if (v == 4) k_norm_rotary<TX, TY, 4, true, 1, BWD, AHEAD><<<grid, kThreadsNorm, lds, s>>>(a);
    else k_norm_rotary<TX, TY, 2, true, 2, BWD, AHEAD><<<grid, kThreadsNorm, lds, s>>>(a);
  } else {
    if constexpr (sizeof(TX) + sizeof(TY) < 8)
      if (v == 8) return (void)(k_norm_rotary<TX, TY, 8, false, 1, BWD, AHEAD><<<grid, kThreadsNorm, lds, s>>>(a));
    if (v == 4) k_norm_rotary<TX, TY, 4, false, 1, BWD, AHEAD><<<grid, kThreadsNorm, lds, s>>>(a);
    else k_norm_rotary<TX, TY, 2, false, 2, BWD, AHEAD><<<grid, kThreadsNorm, lds, s>>>(a);
  }
}
template <typename TX, typename TY>
void run_types(const NormArgs& a, int v, bool halves, bool backward, dim3 grid, size_t lds, hipStream_t s) {
  if (!backward) run_form<TX, TY, false, 2>(a, v, halves, grid, 0, s);
  else if (a.heads_a_thread > 1) run_form<TX, TY, true, 2>(a, v, halves, grid, lds, s);
  else run_form<TX, TY, true, 1>(a, v, halves, grid, lds, s);
}

// Heads a lane turns with one set of angles, weights and, backward, sums: as many as leave enough threads to keep the
// memory busy (us for Q and K, bf16, 12 heads of 128, with 2^16, 2^17 and 2^18 threads: forward 4680 tokens 14.1, 12.7, 13.7, a
// weight for every head 16.3, 13.3, 14.3, 16 heads of 80, 3000 tokens, 12.6, 10.4, 10.4; backward 4680 tokens 22.6, 23.8, 26.5,
// 1560 tokens 13.4, 13.7, 16.2).
constexpr long long kEnoughForward = 1 << 17, kEnoughBackward = 1 << 16;

}  // namespace

hipError_t launch_norm_rotary(const mrt_rotary& r, float eps, const mrt_norm_tensor* x, int n, const void* const* X,
                              const void* const* dY, void* const* out, float* workspace, hipStream_t s) {
  const bool backward = dY != nullptr;
  NormArgs a;
  a.pairs = r.pairs[0] + r.pairs[1] + r.pairs[2];
  a.end0 = r.pairs[0];
  a.end1 = r.pairs[0] + r.pairs[1];
  a.adjacent = r.layout == MRT_ROTARY_ADJACENT;
  a.d = r.head_dim;
  a.eps = eps;
  a.inv_d = 1.0f / r.head_dim;
  // powers of the ladder's ratio in 64 significant bits, as rotary_turns has them, with one pow for a ladder that is shared
  const long double quarter = (backward ? -2.0L : 2.0L) / 3.14159265358979323846264338327950288L;
  long double at = quarter, ratio = 1;
  for (int axis = 0, p = 0; axis < 3; ++axis) {
    const bool shared = r.ladder == MRT_ROTARY_SHARED;
    if (p == 0 || !shared) {
      if (r.pairs[axis] == 0) continue;
      at = quarter;
      ratio = powl((long double)r.theta, -1.0L / (shared ? a.pairs : r.pairs[axis]));
    }
    for (int i = 0; i < r.pairs[axis]; ++i, at *= ratio) a.quarters[p++] = (double)at;
  }
  NormJoin join;
  join.d = r.head_dim;
  int most_joined = 0;
  for (int i = 0; i < 2; ++i) { join.parts[i] = nullptr; join.dweight[i] = nullptr; join.n[i] = join.heads[i] = 0; }
  int v[2] = {1, 1};
  for (int i = 0; i < n; ++i) v[i] = run_length(r, x[i], X[i], backward ? dY[i] : nullptr, out[i], backward, a.pairs);
  // one launch for both tensors if they have the same types and alignment
  const bool together = n > 1 && x[0].t.x_dtype == x[1].t.x_dtype && x[0].t.y_dtype == x[1].t.y_dtype && v[0] == v[1];
  for (int first = 0; first < n; first += together ? 2 : 1) {
    const int count = together ? 2 : 1, run = v[first];
    a.turned = a.adjacent && run > 1 ? 2 * a.pairs / run : a.pairs / run;
    a.items = a.turned + (r.head_dim - 2 * a.pairs) / run;
    a.lanes = 1;
    while (a.lanes < a.items && a.lanes < 64) a.lanes *= 2;
    const int rows_a_block = kThreadsNorm / a.lanes;
    long long threads = 0;
    int most_heads = 1;
    bool each = false;
    for (int i = 0; i < count; ++i) {
      const mrt_norm_tensor& t = x[first + i];
      threads += (long long)t.t.batch * t.t.f * t.t.h * t.t.w * a.lanes * t.t.heads;
      most_heads = std::max(most_heads, t.t.heads);
      each = each || (backward && t.dweight && t.weight_head);
    }
    a.heads_a_thread = each ? 1 : 16;
    while (a.heads_a_thread > 1 && threads / a.heads_a_thread < (backward ? kEnoughBackward : kEnoughForward)) a.heads_a_thread /= 2;
    if (!each)
      while ((most_heads + a.heads_a_thread - 1) / a.heads_a_thread > (backward ? kMostNormParts : 65535)) a.heads_a_thread *= 2;
    // (runs of one length)
    const int runs_a_row = (most_heads + a.heads_a_thread - 1) / a.heads_a_thread;
    a.heads_a_thread = (most_heads + runs_a_row - 1) / runs_a_row;
    int blocks[2] = {0, 0};
    for (int i = 0; i < count; ++i) {
      const int k = first + i;
      const mrt_norm_tensor& t = x[k];
      const int tokens = t.t.f * t.t.h * t.t.w, runs = (t.t.heads + a.heads_a_thread - 1) / a.heads_a_thread;
      const long long rows = (long long)t.t.batch * tokens;
      blocks[i] = (int)((rows + rows_a_block - 1) / rows_a_block);
      if (backward) blocks[i] = std::min(blocks[i], std::max(1, kMostNormParts / runs));
      a.t[i] = NormTensor{X[k], backward ? dY[k] : nullptr, out[k], t.weight, nullptr, backward ? t.dweight : nullptr,
                          t.t.positions, t.t.position_batch, t.t.position_axis, t.weight ? t.weight_head : 0,
                          t.t.x, t.t.y, backward ? t.dx : t.t.y, t.t.heads, tokens, (int)rows, t.t.h, t.t.w, t.t.frame_offset,
                          t.weight_dtype == MRT_F32, blocks[i], runs};
      if (backward && t.dweight) {
        const bool own = t.weight && t.weight_head;
        a.t[i].parts = workspace;
        join.parts[k] = workspace;
        join.dweight[k] = t.dweight;
        join.heads[k] = own ? t.t.heads : 1;
        join.n[k] = own ? blocks[i] : blocks[i] * runs;
        most_joined = std::max(most_joined, join.heads[k]);
        workspace += (size_t)blocks[i] * runs * r.head_dim;
      }
    }
    if (count == 1) a.t[1] = a.t[0];
    a.split_block = blocks[0];
    const dim3 grid((unsigned)(blocks[0] + blocks[1]), (unsigned)((most_heads + a.heads_a_thread - 1) / a.heads_a_thread));
    const size_t lds = (size_t)rows_a_block * r.head_dim * sizeof(float);
    const bool halves = !a.adjacent, xf = x[first].t.x_dtype == MRT_F32, yf = x[first].t.y_dtype == MRT_F32;
    if (xf && yf) run_types<float, float>(a, run, halves, backward, grid, lds, s);
    else if (xf) run_types<float, __bf16>(a, run, halves, backward, grid, lds, s);
    else if (yf) run_types<__bf16, float>(a, run, halves, backward, grid, lds, s);
    else run_types<__bf16, __bf16>(a, run, halves, backward, grid, lds, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (most_joined > 0) {
    k_norm_join<<<dim3((r.head_dim + 15) / 16, most_joined, 2), 256, 0, s>>>(join);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace mrt
