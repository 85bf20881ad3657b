// Rotary positions with three axes, forward and backward (the turn by the opposite angle).
//
// Every element is read and written once: memory bounds the call (12 heads of 4680 tokens of 128, Q and K, bf16: 57 MB in
// 11.6 us).  A thread owns V consecutive features of a token (in halves: V of the first half and their partners) for a
// run of heads, so that the angles, which all heads share, are formed once a run.  The angle of a pair is kept in turns: position x (turns per position) in 64 bits,
// whose whole part is dropped exactly before the rest goes to 32 bits.  So no position is too far (a 32-bit angle
// at position 10^6 is off by 0.06 radians), and nothing is read from a table.
#include "mrt_rotary.hpp"
#include "mrt_rotary_rows.hpp"
#include "mrt_bf16_tiles.hpp"

namespace mrt {

namespace {

constexpr int kThreadsRot = 256;

struct RotaryTensor {
  const void* x;
  void* y;
  const int* positions;
  long long pos_batch, pos_axis;
  mrt_strides xs, ys;
  int heads, tokens, rows;      // rows: batch x tokens
  int h, w, frame0;
};
struct RotaryArgs {
  RotaryTensor t[2];
  double turns[kMostPairs];     // of a pair, per position; negative for the inverse
  int end0, end1, pairs;        // first pair of the second and the third axis, all pairs
  int chunks, turned;           // work items of a token, those of them that turn (the others copy)
  int split_block;              // first block of the second tensor
  int heads_a_thread, adjacent;
};

// V: elements of one access.  HALVES: a thread's accesses are V elements and their V partners; with V = 1 these may
// be adjacent ones, in rows whose pairs are not aligned.  AHEAD: heads whose loads are in flight at once.
template <typename TX, typename TY, int V, bool HALVES>
__global__ __launch_bounds__(kThreadsRot) void k_rotary(const RotaryArgs a) {
  constexpr int NP = HALVES ? V : V / 2, N = HALVES ? 2 * V : V, AHEAD = 4;
  const bool second = (int)blockIdx.x >= a.split_block;
  const RotaryTensor& t = a.t[second];
  const int block = blockIdx.x - (second ? a.split_block : 0);
  const int local = threadIdx.x / a.chunks, chunk = threadIdx.x - local * a.chunks, rows_a_block = kThreadsRot / a.chunks;
  const long long row_l = (long long)block * rows_a_block + local;
  const int h0 = blockIdx.y * a.heads_a_thread, h1 = h0 + a.heads_a_thread < t.heads ? h0 + a.heads_a_thread : t.heads;
  if (local >= rows_a_block || row_l >= t.rows || h0 >= h1) return;
  const int row = (int)row_l, b = row / t.tokens, token = row - b * t.tokens;
  const TX* x = (const TX*)t.x + b * t.xs.batch + token * t.xs.token + h0 * t.xs.head;
  TY* y = (TY*)t.y + b * t.ys.batch + token * t.ys.token + h0 * t.ys.head;
  if (chunk >= a.turned) {               // features that no pair takes
    const int f = 2 * a.pairs + V * (chunk - a.turned);
    for (int h = h0; h < h1; ++h, x += t.xs.head, y += t.ys.head) {
      float v[V];
      load_run<TX, V>(x + f, v);
      store_run<TY, V>(y + f, v);
    }
    return;
  }
  const bool next = V == 1 && a.adjacent;
  const int f0 = next ? 2 * chunk : V * chunk, f1 = next ? f0 + 1 : f0 + a.pairs, p0 = HALVES ? V * chunk : f0 / 2;
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
  float cs[NP], sn[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int p = p0 + i, at = p < a.end0 ? pos[0] : p < a.end1 ? pos[1] : pos[2];
    const double turn = at * a.turns[p];
    sincospif(2.0f * (float)(turn - rint(turn)), &sn[i], &cs[i]);
  }
  for (int h = h0; h < h1; h += AHEAD) {
    float v[AHEAD][N];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const TX* at = x + (h + k < h1 ? k : 0) * t.xs.head;
      float u[V];
      load_run<TX, V>(at + f0, u);
#pragma unroll
      for (int e = 0; e < V; ++e) v[k][e] = u[e];
      if constexpr (HALVES) {
        load_run<TX, V>(at + f1, u);
#pragma unroll
        for (int e = 0; e < V; ++e) v[k][V + e] = u[e];
      }
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (h + k >= h1) break;
      TY* at = y + k * t.ys.head;
      float u[V], w[V];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const float x0 = HALVES ? v[k][i] : v[k][2 * i], x1 = HALVES ? v[k][V + i] : v[k][2 * i + 1];
        const float y0 = fmaf(x0, cs[i], -(x1 * sn[i])), y1 = fmaf(x0, sn[i], x1 * cs[i]);
        if constexpr (HALVES) { u[i] = y0; w[i] = y1; }
        else { u[2 * i] = y0; u[2 * i + 1] = y1; }
      }
      store_run<TY, V>(at + f0, u);
      if constexpr (HALVES) store_run<TY, V>(at + f1, w);
    }
    x += AHEAD * t.xs.head;
    y += AHEAD * t.ys.head;
  }
}

// Elements that the rows of a tensor can be moved by at once.
int run_length(const mrt_rotary& r, const mrt_rotary_tensor& x, const void* X, const void* Y, int pairs) {
  for (int v = 8; v > 1; v /= 2) {
    bool ok = r.head_dim % v == 0 && (r.layout == MRT_ROTARY_ADJACENT ? 2 * pairs : pairs) % v == 0;
    const mrt_strides* st[2] = {&x.x, &x.y};
    const void* at[2] = {X, Y};
    for (int k = 0; ok && k < 2; ++k) {
      const size_t size = (k ? x.y_dtype : x.x_dtype) == MRT_F32 ? 4 : 2, bytes = v * size < 16 ? v * size : 16;
      ok = (uintptr_t)at[k] % bytes == 0 && st[k]->token * size % bytes == 0 && st[k]->head * size % bytes == 0 &&
           st[k]->batch * size % bytes == 0;
    }
    if (ok) return v;
  }
  return 1;
}

template <typename TX, typename TY>
void run_types(const RotaryArgs& a, int v, bool halves, dim3 grid, hipStream_t s) {
  if (v == 1) k_rotary<TX, TY, 1, true><<<grid, kThreadsRot, 0, s>>>(a);
  else if (halves) {
    if (v == 8) k_rotary<TX, TY, 8, true><<<grid, kThreadsRot, 0, s>>>(a);
    else if (v == 4) k_rotary<TX, TY, 4, true><<<grid, kThreadsRot, 0, s>>>(a);
    else k_rotary<TX, TY, 2, true><<<grid, kThreadsRot, 0, s>>>(a);
  } else {
    if (v == 8) k_rotary<TX, TY, 8, false><<<grid, kThreadsRot, 0, s>>>(a);
    else if (v == 4) k_rotary<TX, TY, 4, false><<<grid, kThreadsRot, 0, s>>>(a);
    else k_rotary<TX, TY, 2, false><<<grid, kThreadsRot, 0, s>>>(a);
  }
}

// Heads a thread turns with one set of angles: as many as leave enough threads to keep the memory busy, a wave on each
// SIMD (us for Q and K, bf16, heads of 128, with 2^16, 2^18 and 2^20 threads: 12 heads of 1560 tokens 5.2, 6.5, 9.2, of
// 4680 tokens 11.6, 11.6, 21.3, of 14040 tokens 28 each; 40 heads of 300 tokens 4.5, 6.7, 6.5).
constexpr long long kEnoughThreads = 1 << 16;

}  // namespace

hipError_t launch_rotary(const mrt_rotary& r, const mrt_rotary_tensor* x, int n, const void* const* X, void* const* Y,
                         bool inverse, hipStream_t s) {
  RotaryArgs a;
  a.pairs = r.pairs[0] + r.pairs[1] + r.pairs[2];
  a.end0 = r.pairs[0];
  a.end1 = r.pairs[0] + r.pairs[1];
  a.adjacent = r.layout == MRT_ROTARY_ADJACENT;
  rotary_turns(r, inverse, a.turns);
  // one launch for both tensors if they have the same types and alignment
  const int v0 = run_length(r, x[0], X[0], Y[0], a.pairs), v1 = n > 1 ? run_length(r, x[1], X[1], Y[1], a.pairs) : v0;
  const bool together = n > 1 && x[0].x_dtype == x[1].x_dtype && x[0].y_dtype == x[1].y_dtype && v0 == v1;
  for (int first = 0; first < n; first += together ? 2 : 1) {
    const int count = together ? 2 : 1, v = first ? v1 : v0;
    a.turned = a.adjacent && v > 1 ? 2 * a.pairs / v : a.pairs / v;
    a.chunks = a.turned + (r.head_dim - 2 * a.pairs) / v;
    const int rows_a_block = kThreadsRot / a.chunks;
    long long blocks[2] = {0, 0}, most_heads = 1, threads = 0;
    for (int i = 0; i < count; ++i) {
      const mrt_rotary_tensor& t = x[first + i];
      const int tokens = t.f * t.h * t.w;
      a.t[i] = RotaryTensor{X[first + i], Y[first + i], t.positions, t.position_batch, t.position_axis, t.x, t.y,
                            t.heads, tokens, t.batch * tokens, t.h, t.w, t.frame_offset};
      blocks[i] = ((long long)a.t[i].rows + rows_a_block - 1) / rows_a_block;
      if (t.heads > most_heads) most_heads = t.heads;
      threads += (long long)a.t[i].rows * a.chunks * t.heads;
    }
    if (count == 1) a.t[1] = a.t[0];
    a.split_block = (int)blocks[0];
    a.heads_a_thread = 16;
    while (a.heads_a_thread > 1 && threads / a.heads_a_thread < kEnoughThreads) a.heads_a_thread /= 2;
    // (blocks in y are at most 65535: more heads than that go to a thread each)
    while ((most_heads + a.heads_a_thread - 1) / a.heads_a_thread > 65535) a.heads_a_thread *= 2;
    const dim3 grid((unsigned)(blocks[0] + blocks[1]), (unsigned)((most_heads + a.heads_a_thread - 1) / a.heads_a_thread));
    const bool halves = !a.adjacent;
    const bool xf = x[first].x_dtype == MRT_F32, yf = x[first].y_dtype == MRT_F32;
    if (xf && yf) run_types<float, float>(a, v, halves, grid, s);
    else if (xf) run_types<float, __bf16>(a, v, halves, grid, s);
    else if (yf) run_types<__bf16, float>(a, v, halves, grid, s);
    else run_types<__bf16, __bf16>(a, v, halves, grid, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mrt
