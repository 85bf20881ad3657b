// Backward pass of the dense softmax attention on the bf16 matrix unit (formulas: mrt_dense_train.hpp).
//
// No atomics, two kinds of workgroups in one launch: those of the gradients of the queries own queries and stream the keys,
// those of the keys own keys and stream the queries of every head that reads them.  Seven products where one kind would
// form five; but that one has to add to dQ from every key tile, in an order that changes, or to write and read as many
// partial arrays as there are key tiles (half a gigabyte each way for 12 heads of 4680 tokens).  A small launch before it
// leaves what both need of a row, -log2(e) lse and -delta.  (The two kinds in launches of their own, the first of which
// left these: us of a call, two launches | one: one head of 4680 tokens 86 | 68, 12 of 1560 tokens 105 | 87, 40 of 1800
// tokens 299 | 269, batch of 3, 4 heads of 782 tokens of 64 features 42 | 28, 12 heads of 4680 tokens 444 | 445, 425 with
// two workgroups to a tile of queries, which the launch of one kind did not gain by.)
//
// A wave owns 32 rows: their operands and gradients stay in registers, the streamed rows pass through an LDS ring 32 a
// step, loaded by instructions that write LDS directly, several steps ahead.  Logits have the streamed rows on the M
// side and the wave's rows on the N side of a product, so that weights, packed to bf16, are as they stand the operand
// of the second products, whose other operand is the streamed tile read transposed.
//
// What bounds the launch is power: a wave's 32 rows take a kilobyte of LDS reads for every 32768 operations, and at
// that ratio the card's clock falls until bare products reach about 1400 TFLOP/s (32 x 32 tiles) or 1550 (16 x 16),
// where products from registers reach 1670 and 1950 and a large library product 1355.  Vector instructions hardly run
// beside another wave's 16 x 16 products and half hide behind a wave's own; beside 32 x 32 products of another wave they
// run whole.  So a tile of queries, which has the registers for the logits of two steps, forms the weights of one step
// between its own products of the next, 16 x 16 tiles; a tile of keys, which has not, takes 32 x 32 tiles and leaves it
// to the two workgroups of a compute unit to be in different phases.  (Waves of 64 rows, one to a
// SIMD, halve the LDS reads, but what does not fit 256 registers moves between the two halves of the register file:
// 1.2 to 1.8 times as long.)
#include "mrt_dense_train.hpp"
#include "mrt_bf16_tiles.hpp"


namespace mrt {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((address_space(3))) void lds_void;

__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// Global memory -> LDS, zeros from `bytes` on: lane i's SIZE bytes from base + voff to LDS address at + SIZE i.  Written
// as instructions without a result: to the compiler, which would wait for every load in flight before the next
// transposed read, they touch no register and no counter; wait_and_meet does the waiting.
__device__ inline u32x4 rows_at(const void* base, unsigned bytes) {
  const unsigned long long at = (unsigned long long)base;
  return u32x4{(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)at), (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32)) & 0xffffu,
               (unsigned)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}
// (M0 holds the LDS address; it is put back, because the compiler may keep something there)
__device__ inline void load_lds_16B(u32x4 rows, unsigned at, unsigned voff) {
  unsigned m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(at), "v"(voff), "s"(rows) : "memory");
}
__device__ inline void load_lds_4B(u32x4 rows, unsigned at, unsigned voff) {
  unsigned m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dword %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(at), "v"(voff), "s"(rows) : "memory");
}
// waits for this wave's loads but the last N, and for its LDS reads, then for the other waves
template <int N> __device__ inline void wait_and_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 32 * kWaves;     // two workgroups to a compute unit
constexpr int kStep = 32;          // streamed rows a step
constexpr int kSlots = 4;          // steps in the LDS ring: two or three in use, the others on their way
template <int D> constexpr int kTileBytes = kStep * D * 2;

extern __shared__ __attribute__((aligned(1024))) char bwd_lds[];

// The streamed rows of two arrays (and, KV, the row statistics of the queries) on their way through the LDS ring.
//
// A tile of 32 rows of D bf16 is not padded, because an instruction writes 64 consecutive 16-byte pieces: piece p of row
// r lies at p ^ swz(r), whichever suits the reads (the lane that writes a piece fetches the one that belongs there).
template <int D, bool KV>
struct Stream {
  static constexpr int RB = 2 * D, PIECES = D / 8, SLOT = 2 * kTileBytes<D> + (KV ? 256 : 0), RING = kSlots * SLOT;
  static constexpr int TILE_LOADS = kTileBytes<D> / 1024, LOADS = 2 * TILE_LOADS / kWaves;   // of one array's tile; a wave's share of both
  static constexpr int PERSTEP = LOADS + (KV ? 1 : 0);                                  // loads a wave has in flight for a step
  static_assert(TILE_LOADS % kWaves == 0, "whole loads, of one array each");
  const u16 *a, *b;
  const float* stats;
  long long at, bt, anext, bnext;       // elements from row to row, and from the end of a head's rows to the next head's
  int steps, left, left0, snext;
  unsigned to, lds0, arow, brow;
  int wave, lane;

  // n steps of rows from `row` on, `left` of them; KV: then left0 rows of the next head
  __device__ inline void start(const u16* a_, long long at_, const u16* b_, long long bt_, const float* stats_, int n, int left_, int wave_, int lane_) {
    a = a_; b = b_; at = at_; bt = bt_; stats = stats_;
    steps = n; left = left_; wave = wave_; lane = lane_;
    arow = (unsigned)at * 2u; brow = (unsigned)bt * 2u;
    to = 0;
    lds0 = (unsigned)(unsigned long long)(const lds_void*)bwd_lds;
  }
  template <typename Swz>
  __device__ inline void issue(Swz swz) {
    const unsigned rows = steps > 0 ? (left < kStep ? left : kStep) : 0;
    const u32x4 ra = rows_at(a, rows ? (rows - 1) * arow + RB : 0), rb = rows_at(b, rows ? (rows - 1) * brow + RB : 0);
    const unsigned slot = __builtin_amdgcn_readfirstlane(lds0 + to);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const bool of_b = j * kWaves >= TILE_LOADS;
      const int s = (j * kWaves + wave) % TILE_LOADS * 64 + lane, row = s / PIECES, piece = (s % PIECES) ^ swz(row);
      load_lds_16B(of_b ? rb : ra, slot + (j * kWaves + wave) * 1024, row * (of_b ? brow : arow) + piece * 16);
    }
    if constexpr (KV) {       // (every wave writes the same 256 bytes: all wait for the same number of loads)
      load_lds_4B(rows_at(stats, rows ? 256 : 0), slot + 2 * kTileBytes<D>, lane * 4);
      stats += 64;
    }
    --steps;
    a += kStep * at;
    b += kStep * bt;
    left -= kStep;
    if (KV && left <= 0 && steps > 0) {
      a += anext;
      b += bnext;
      stats += snext;
      left = left0;
    }
    to = to + SLOT == RING ? 0 : to + SLOT;
  }
  static __device__ inline int after(int slot) { return slot + SLOT == RING ? 0 : slot + SLOT; }
};

// Unit of work of a workgroup: a tile of a (batch, head)'s own rows and one of `parts` runs of the streamed ones.
// Where every query sees every key (no mask, or a chunk against its cache) every XCD gets a contiguous run of units, so that
// those that stream the same rows share its L2; under a mask, where tiles differ in length, the longest go first.  (The
// cache of 32760 keys in the second order 2687 us instead of 2686, of 64 features 1580 instead of 1576, one frame of 1560
// tokens and 3 heads against 8 frames 129 instead of 127: that order is for the calls it is meant for.)
struct Unit {
  int bh, tile, part;
};
__device__ inline Unit unit_of(const DenseBwd& p, int unit, int n_heads, int tiles, int parts, bool last_first) {
  const int total = n_heads * tiles * parts;
  Unit u;
  if (dense_last_key(p, 0, p.Nkv) == p.Nkv) {
    const int xcd = unit & 7;
    unit = xcd * (total >> 3) + (xcd < (total & 7) ? xcd : (total & 7)) + (unit >> 3);
    u.tile = unit % tiles;
    unit /= tiles;
    u.part = unit % parts;
    u.bh = unit / parts;
  } else {
    u.bh = unit % n_heads;
    unit /= n_heads;
    u.part = unit % parts;
    u.tile = unit / parts;
    if (last_first) u.tile = tiles - 1 - u.tile;
  }
  return u;
}

// A row's four consecutive features as bf16, or in fp32 among the parts.
template <bool PART>
__device__ inline void put4(u16* row, float* part, int f, f32x4 x) {
  if constexpr (PART) *(f32x4*)(part + f) = x;
  else *(bf16x4*)(row + f) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
}

// ---- what both need of a row ----------------------------------------------------------------------
// -log2(e) lse (-infinity where a row sees no key: weights of zero) and -delta of 32 rows a workgroup, eight threads a row;
// rows behind the last one as such that see no key.  Memory bounds it (12 heads of 4680 tokens 7 us;
// 32 heads of 1531 causal tokens 8.7, 6.6 without what follows).
//
// delta = O . dO.  The forward call rounded O to bf16, and where a row sees few keys that is the largest error of its dS:
// all of it has the same sign, beside roundings of dS that do not (gradients of 10 causal tokens 3.2e-3 of the 2-norm off
// instead of 2.4e-3, of 16 queries over 4 keys 2.8e-3 instead of 2.2e-3, of 1531 causal tokens 2.48e-3 instead of 2.36e-3).
// So rows that see at most a tile of keys for each wave form delta as the sum of P dP.
constexpr int kFewKeys = 32 * kWaves;
template <int D>
__global__ __launch_bounds__(kThreads) void k_bf16_dense_bwd_stats(DenseBwd p, int nqb) {
  constexpr int KS = D / 16;
  // (the first queries of all heads, which see the fewest keys and take longest, come first)
  const int heads = p.B * p.H, bh = blockIdx.x % heads, block = blockIdx.x / heads;
  const long long tile = (long long)bh * nqb + block;
  const int q0 = 32 * block, b = bh / p.H, hd = bh - b * p.H, kvh = hd / p.group;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const u16* dOp = (const u16*)p.dO + b * p.dout.batch + hd * p.dout.head;
  float* stats = p.stats + tile * 64;
  const int keys = __builtin_amdgcn_readfirstlane(dense_seen_keys(p, b)), q_last = q0 + 31 < p.Nq ? q0 + 31 : p.Nq - 1;
  const int most = dense_last_key(p, q_last, keys);
  auto negative_lse = [&](int q) {
    const float l = q < p.Nq ? p.lse[(long long)bh * p.Nq + q] : -INFINITY;
    return l == -INFINITY ? -INFINITY : -kLog2e * l;
  };
  if (most > 0 && most <= kFewKeys) {
    __shared__ float sums[kWaves][32];
    const int hi = lane >> 5, c = lane & 31, q = q0 + c, k0 = 32 * wave, lim = q < p.Nq ? dense_last_key(p, q, keys) : 0;
    const long long qr = q < p.Nq ? q : p.Nq - 1, kr = k0 + c < most ? k0 + c : most - 1;
    const u16* Qp = (const u16*)p.Q + b * p.q.batch + hd * p.q.head + qr * p.q.token + 8 * hi;
    const u16* Gp = dOp + qr * p.dout.token + 8 * hi;
    const u16* Kp = (const u16*)p.K + b * p.k.batch + kvh * p.k.head + kr * p.k.token + 8 * hi;
    const u16* Vp = (const u16*)p.V + b * p.v.batch + kvh * p.v.head + kr * p.v.token + 8 * hi;
    const float nl = negative_lse(q), scale2 = p.scale * kLog2e;
    f32x16 s = {}, dp = {};         // rows: keys k0 + 8 (r >> 2) + 4 hi + (r & 3); columns: queries
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      s = mfma32(ld_global_16B(Kp + 16 * ks), ld_global_16B(Qp + 16 * ks), s);
      dp = mfma32(ld_global_16B(Vp + 16 * ks), ld_global_16B(Gp + 16 * ks), dp);
    }
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
      stats[c] = nl;
      stats[32 + c] = -((sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]));
    }
    return;
  }
  constexpr int PER = D / 64;            // 16-byte pieces of a row a thread takes
  const int r = tid >> 3, q = q0 + r;
  const long long qr = q < p.Nq ? q : p.Nq - 1;
  const u16* Op = (const u16*)p.O + b * p.o.batch + hd * p.o.head + qr * p.o.token + 8 * (tid & 7);
  dOp += qr * p.dout.token + 8 * (tid & 7);
  const float nl = negative_lse(q);
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const bf16x8 x = ld_global_16B(Op + 64 * j), y = ld_global_16B(dOp + 64 * j);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf((float)x[e], (float)y[e], sum);
  }
  sum = row8_sum(sum);
  if ((tid & 7) == 0) {
    stats[r] = nl;
    stats[32 + r] = q < p.Nq ? -sum : 0.f;
  }
}

// ---- queries -----------------------------------------------------------------------------------
// Two tiles of 16 queries a wave.  A step's products run in this order: A, the logits and dO V^T of the next step's keys;
// B, dQ^T += K^T dS of this step.  Between the products of A stand the exponentials and gradients of this step's logits.
template <int D, bool PART>
__device__ __forceinline__ void bwd_queries(const DenseBwd& p, int unit) {
  constexpr int NT = 2, KS = D / 32, FT = D / 16, RB = 2 * D;
  using S = Stream<D, false>;
  // rows are swizzled by pairs of pieces: the sixteen rows x two pairs a 16-byte read takes at once (rows 0-3 and 12-15
  // of one piece, 4-11 of the next, and so on) and the eight rows x one pair of a transposed read lie on all 64 banks
  auto swz = [](int row) { return D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; };
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int parts = PART ? p.parts_q : 1;
  const Unit u = unit_of(p, unit, p.B * p.H, (p.Nq + kRows - 1) / kRows, parts, true);
  const int b = u.bh / p.H, hd = u.bh - b * p.H, kvh = hd / p.group;
  const int q0 = u.tile * kRows, q_last = q0 + kRows < p.Nq ? q0 + kRows - 1 : p.Nq - 1;
  const int keys = __builtin_amdgcn_readfirstlane(dense_seen_keys(p, b)), k_end = dense_last_key(p, q_last, keys), nqb = (p.Nq + 31) >> 5;
  const int all = (k_end + kStep - 1) / kStep;
  const int i0 = PART ? (int)((long long)all * u.part / parts) : 0, i1 = PART ? (int)((long long)all * (u.part + 1) / parts) : all;

  S st;
  st.start((const u16*)p.K + b * p.k.batch + kvh * p.k.head + (long long)kStep * i0 * p.k.token, p.k.token,
           (const u16*)p.V + b * p.v.batch + kvh * p.v.head + (long long)kStep * i0 * p.v.token, p.v.token, nullptr,
           i1 - i0, k_end - kStep * i0, wave, lane);
#pragma unroll
  for (int j = 0; j < kSlots - 1; ++j) st.issue(swz);

  // the wave's queries
  const u16* Qp = (const u16*)p.Q + b * p.q.batch + hd * p.q.head;
  const u16* dOp = (const u16*)p.dO + b * p.dout.batch + hd * p.dout.head;
  const int qw = q0 + 16 * NT * wave;
  bf16x8 qf[NT][KS], of[NT][KS];
  float nlse[NT], ndelta[NT];          // -log2(e) lse, -delta
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int q = qw + 16 * t + c;
    const long long r = q < p.Nq ? q : p.Nq - 1;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[t][ks] = ld_global_16B(Qp + r * p.q.token + 32 * ks + 8 * g);
      of[t][ks] = ld_global_16B(dOp + r * p.dout.token + 32 * ks + 8 * g);
    }
    const float* stats = p.stats + ((long long)u.bh * nqb + (r >> 5)) * 64 + (r & 31);
    nlse[t] = stats[0];
    ndelta[t] = stats[32];
  }
  const float scale2 = p.scale * kLog2e;
  f32x4 dq[NT][FT];    // dQ^T
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int f = 0; f < FT; ++f) dq[t][f] = f32x4{0.f, 0.f, 0.f, 0.f};

  // where a lane reads the first of its operands of a tile; the others differ in bits (^) and rows (+)
  const int s4 = c >> 2, trow = 4 * g + s4;
  const int row_at = c * RB + (swz(c) ^ g) * 16, tr_at = trow * RB + swz(trow) * 16 + 8 * (c & 3);
  auto row_op = [&](int at, int ks, int m) { return *(const bf16x8*)(bwd_lds + (at ^ (64 * ks)) + 16 * m * RB); };
  auto tr_op = [&](int at, int f) {
    const u16* q = (const u16*)(bwd_lds + (at ^ (32 * f)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(ld_lds_tr(q), ld_lds_tr(q + 16 * D), 0, 1, 2, 3, 4, 5, 6, 7));
  };

  f32x4 sv[2][NT][2], dp[2][NT][2];     // logits and dO V^T of two steps in turn
  bf16x8 db[NT];
  // operands are read from LDS three ahead of their products, over the end of a step too
  constexpr int NA = 4 * KS, OPS = NA + FT;
  static_assert(OPS % 4 == 0, "operands keep their registers from step to step");
  bf16x8 op[4];
  auto read_op = [&](int i, int next, int slot) {
    if (i < NA) op[i & 3] = row_op(i & 1 ? next + kTileBytes<D> : next, i >> 2, (i >> 1) & 1);
    else op[i & 3] = tr_op(slot, i - NA);
  };
  auto product_a = [&](auto buf, int i, int t) {
    constexpr int B = decltype(buf)::value;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const int ks = i >> 2, m = (i >> 1) & 1;
    if ((i & 1) == 0) sv[B][t][m] = mfma(op[i & 3], qf[t][ks], ks == 0 ? zero : sv[B][t][m]);
    else dp[B][t][m] = mfma(op[i & 3], of[t][ks], ks == 0 ? zero : dp[B][t][m]);
  };
  auto soften = [&](auto buf, int e) {
    constexpr int B = decltype(buf)::value;
    const int t = e >> 3, m = (e >> 2) & 1, r = e & 3;
    dp[B][t][m][r] = exp2_fast(fmaf(sv[B][t][m][r], scale2, nlse[t])) * (dp[B][t][m][r] + ndelta[t]);
    if ((e & 7) == 7) db[t] = pack8(dp[B][t][0], dp[B][t][1]);
  };
  const int free_keys = dense_last_key(p, q0, keys);       // every query of the workgroup sees these
  int row = kStep * i0, slot = 0, next = S::SLOT;
  auto step = [&](auto buf, bool live) {
    constexpr int B = decltype(buf)::value;
    const std::integral_constant<int, 1 - B> other;
    // some query does not see the step whole, or there is no such step (an odd number of them)
    if (!live || row + kStep > free_keys) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int q = qw + 16 * t + c, lim = live ? dense_last_key(p, q < p.Nq ? q : p.Nq - 1, keys) : 0;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (row + 16 * m + 4 * g + r >= lim) { sv[B][t][m][r] = -INFINITY; dp[B][t][m][r] = 0.f; }
      }
    }
    const int at = slot + tr_at, nt = next + row_at;
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      read_op(i + 3, nt, at);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        product_a(other, i, t);
        constexpr int EVERY = NA * NT / (8 * NT);
        if ((i * NT + t) % EVERY == 0) soften(buf, (i * NT + t) / EVERY);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // (the ring holds this step, the next one and the one after, which the first reads below are for)
    wait_and_meet<(kSlots - 4) * S::PERSTEP>();
    st.issue(swz);
    const int then = S::after(next), nnt = then + row_at;
#pragma unroll
    for (int i = NA; i < OPS; ++i) {
      if (i + 3 < OPS) read_op(i + 3, nt, at);
      else read_op(i + 3 - OPS, nnt, at);
#pragma unroll
      for (int t = 0; t < NT; ++t) dq[t][i - NA] = mfma(op[i & 3], db[t], dq[t][i - NA]);
      __builtin_amdgcn_sched_barrier(0);
    }
    slot = next;
    next = then;
    row += kStep;
  };
  wait_and_meet<(kSlots - 3) * S::PERSTEP>();
  if (i0 < i1) {
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      read_op(i, row_at, 0);
#pragma unroll
      for (int t = 0; t < NT; ++t) product_a(even, i, t);
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) read_op(i, next + row_at, 0);
    for (int i = i0; i < i1; i += 2) {
      step(even, true);
      step(odd, i + 1 < i1);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing is on its way to LDS when the workgroup leaves it

#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const long long q = qw + 16 * t + c;
    if (q >= p.Nq) continue;
    u16* to = (u16*)p.dQ + b * p.dq.batch + hd * p.dq.head + q * p.dq.token + 4 * g;
    float* part = p.pq + (((long long)u.part * p.B * p.H + u.bh) * p.Nq + q) * D + 4 * g;
#pragma unroll
    for (int f = 0; f < FT; ++f) put4<PART>(to, part, 16 * f, dq[t][f] * p.scale);
  }
}

// ---- keys --------------------------------------------------------------------------------------
// One tile of 32 keys a wave.  A step is a vector phase (weights and gradients of the logits), which runs beside the
// matrix phase of the other workgroup's wave on the SIMD, and a matrix phase (what these give to dV^T and dK^T, then the
// logits and dO V^T of the next step's queries).
template <int D, bool PART>
__device__ __forceinline__ void bwd_keys(const DenseBwd& p, int unit) {
  constexpr int KS = D / 16, FT = D / 32, RB = 2 * D, AHEAD = 3;
  using S = Stream<D, true>;
  // sixteen rows that agree in a piece lie on all 64 banks (those a 16-byte read takes at once: 0-3, 12-15 and 20-27 of a
  // tile, and the other sixteen), and so do four consecutive rows of four pieces (a transposed read).  Rows 8 apart
  // differ in bit 1, rows 16 apart in nothing.
  auto swz = [](int row) { return D == 128 ? (row & 3) << 2 | ((row >> 2) & 3) : (row & 2) << 1 | ((row >> 2) & 3); };
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, hi = lane >> 5, c = lane & 31;
  const int parts = PART ? p.parts_kv : 1;
  const Unit u = unit_of(p, unit, p.B * p.KH, (p.Nkv + kRows - 1) / kRows, parts, false);
  const int b = u.bh / p.KH, hd = u.bh - b * p.KH;
  const int k0 = u.tile * kRows, k_last = k0 + kRows < p.Nkv ? k0 + kRows - 1 : p.Nkv - 1;
  const int keys = __builtin_amdgcn_readfirstlane(dense_seen_keys(p, b)), nqb = (p.Nq + 31) >> 5;
  const int q_first = dense_first_query(p, k0) & ~(kStep - 1);      // of every head that reads these keys
  const int per_head = k0 < keys && q_first < p.Nq ? (p.Nq - q_first + kStep - 1) / kStep : 0, all = per_head * p.group;
  const int i0 = PART ? (int)((long long)all * u.part / parts) : 0, i1 = PART ? (int)((long long)all * (u.part + 1) / parts) : all;

  S st;
  int row;           // of the step in hand
  {
    const int gh = per_head > 0 ? i0 / per_head : 0, hq = hd * p.group + gh;
    row = q_first + kStep * (i0 - gh * per_head);
    st.start((const u16*)p.Q + b * p.q.batch + hq * p.q.head + row * p.q.token, p.q.token,
             (const u16*)p.dO + b * p.dout.batch + hq * p.dout.head + row * p.dout.token, p.dout.token,
             p.stats + ((long long)(b * p.H + hq) * nqb + (row >> 5)) * 64, i1 - i0, p.Nq - row, wave, lane);
    st.anext = p.q.head - (long long)per_head * kStep * p.q.token;
    st.bnext = p.dout.head - (long long)per_head * kStep * p.dout.token;
    st.snext = 64 * (nqb - per_head);
    st.left0 = p.Nq - q_first;
  }
#pragma unroll
  for (int j = 0; j < kSlots - 1; ++j) st.issue(swz);

  // the wave's keys
  const int kw = k0 + 32 * wave, key = kw + c;
  const long long kr = key < p.Nkv ? key : p.Nkv - 1;
  const u16* Kp = (const u16*)p.K + b * p.k.batch + hd * p.k.head + kr * p.k.token;
  const u16* Vp = (const u16*)p.V + b * p.v.batch + hd * p.v.head + kr * p.v.token;
  bf16x8 kf[KS], vf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = ld_global_16B(Kp + 16 * ks + 8 * hi);
    vf[ks] = ld_global_16B(Vp + 16 * ks + 8 * hi);
  }
  const float scale2 = p.scale * kLog2e;
  f32x16 dv[FT], dk[FT];    // dV^T, dK^T
#pragma unroll
  for (int f = 0; f < FT; ++f) dv[f] = dk[f] = f32x16{};

  // where a lane reads the first of its operands of a tile; the others differ in bits (^) and rows (+)
  const int G = lane >> 4, s = lane & 15, trow = 4 * hi + (s >> 2);
  const int row_at = c * RB + (swz(c) ^ hi) * 16, tr_at = trow * RB + ((2 * (G & 1) + ((s >> 1) & 1)) ^ swz(trow)) * 16 + 8 * (s & 1);
  auto row_op = [&](int at, int ks) { return *(const bf16x8*)(bwd_lds + (at ^ (32 * ks))); };
  auto tr_op = [&](int at, int f, int kk) {
    const char* lo = bwd_lds + (at ^ (64 * f)) + 16 * kk * RB;
    const char* up = bwd_lds + (at ^ (64 * f + 32)) + (16 * kk + 8) * RB;
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(ld_lds_tr((const u16*)lo), ld_lds_tr((const u16*)up), 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto stats_at = [&](int slot, int which, int j) { return *(const f32x4*)(bwd_lds + slot + 2 * kTileBytes<D> + 128 * which + 32 * j + 16 * hi); };

  f32x16 sv, dp;
  bf16x8 pb[2], db[2];
  // The matrix phase.  Operands are read from LDS AHEAD ahead of their products, in this fixed order.
  constexpr int N1 = 2 * FT, NG = 2 * N1, OPS = NG + 2 * KS;
  bf16x8 op[OPS];
  auto read_op = [&](int i, int at, int nt) {
    if (i < N1) op[i] = tr_op(at + kTileBytes<D>, i % FT, i / FT);
    else if (i < NG) op[i] = tr_op(at, (i - N1) % FT, (i - N1) / FT);
    else op[i] = row_op((i - NG) & 1 ? nt + kTileBytes<D> : nt, (i - NG) / 2);
  };
  auto matrix = [&](int slot, int next, int from) {
    const int at = slot + tr_at, nt = next + row_at;
#pragma unroll
    for (int i = 0; i < OPS; ++i)
      if (i >= from && i < from + AHEAD) read_op(i, at, nt);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < OPS; ++i) {
      if (i < from) continue;
      if (i + AHEAD < OPS) read_op(i + AHEAD, at, nt);
      if (i == from ? i == NG : i == NG - 1) {          // the sums of dO V^T begin with -delta
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 x = stats_at(next, 1, j);
#pragma unroll
          for (int r = 0; r < 4; ++r) dp[4 * j + r] = x[r];
        }
      }
      if (i < N1) dv[i % FT] = mfma32(op[i], pb[i / FT], dv[i % FT]);
      else if (i < NG) dk[(i - N1) % FT] = mfma32(op[i], db[(i - N1) / FT], dk[(i - N1) % FT]);
      else if (((i - NG) & 1) == 0) sv = mfma32(op[i], kf[(i - NG) / 2], i == NG ? f32x16{} : sv);
      else dp = mfma32(op[i], vf[(i - NG) / 2], dp);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // The vector phase, of the step in `slot` whose queries begin at `row`.
  const int free_from = p.cc ? dense_first_query(p, k_last) : 0;       // every key of the workgroup is seen from here on
  auto soften = [&](int row, int slot) {
    f32x4 nl[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) nl[j] = stats_at(slot, 0, j);
    if (row < free_from) {
      const int lim = dense_first_query(p, (int)kr);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (row + 8 * (r >> 2) + 4 * hi + (r & 3) < lim) { sv[r] = -INFINITY; dp[r] = 0.f; }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float w = exp2_fast(fmaf(sv[r], scale2, nl[r >> 2][r & 3]));
      pb[r >> 3][r & 7] = (__bf16)w;
      db[r >> 3][r & 7] = (__bf16)(w * dp[r]);
    }
  };

  int left_steps = per_head - (per_head > 0 ? i0 % per_head : 0);
  wait_and_meet<(kSlots - 2) * S::PERSTEP>();
  if (i0 < i1) matrix(0, 0, NG);
  for (int i = i0, slot = 0; i < i1; ++i) {
    const int next = S::after(slot);
    soften(row, slot);
    __builtin_amdgcn_sched_barrier(0);
    wait_and_meet<(kSlots - 3) * S::PERSTEP>();
    st.issue(swz);
    matrix(slot, next, 0);
    slot = next;
    row += kStep;
    if (--left_steps == 0) {
      left_steps = per_head;
      row = q_first;
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing is on its way to LDS when the workgroup leaves it

  if (key >= p.Nkv) return;
  const bool live = key < keys;                 // (the columns of the others may hold anything)
  u16* tk = (u16*)p.dK + b * p.dk.batch + hd * p.dk.head + kr * p.dk.token + 4 * hi;
  u16* tv = (u16*)p.dV + b * p.dv.batch + hd * p.dv.head + kr * p.dv.token + 4 * hi;
  const long long part = (((long long)u.part * p.B * p.KH + u.bh) * p.Nkv + kr) * D + 4 * hi;
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 x, y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = live ? dk[f][4 * j + e] * p.scale : 0.f;
        y[e] = live ? dv[f][4 * j + e] : 0.f;
      }
      put4<PART>(tk, p.pk + part, 32 * f + 8 * j, x);
      put4<PART>(tv, p.pv + part, 32 * f + 8 * j, y);
    }
}

// One launch for both: the key tiles, whose steps are the longer ones, come first.
template <int D, bool PART_Q, bool PART_KV>
__global__ __launch_bounds__(kThreads, 2) void k_bf16_dense_bwd(DenseBwd p, int key_units) {
  const int unit = blockIdx.x;
  if (unit < key_units) bwd_keys<D, PART_KV>(p, unit);
  else bwd_queries<D, PART_Q>(p, unit - key_units);
}

// ---- few queries -------------------------------------------------------------------------------
// Up to 32 rows (the queries of all heads that share a head of keys): one launch reads every key and value once and
// forms all three gradients; memory bounds it.  A wave takes every fourth tile of 32 keys of the workgroup's run, loaded
// into its own part of LDS a tile ahead, with no meeting of waves.  The operands of S = Q K^T in the other order give S^T,
// whose gradients are as they stand the operand of dQ^T += K^T dS^T: sixteen products more, but nothing is moved.  dK
// and dV go through LDS to be stored as whole rows; dQ is summed over the waves, then over the parts.
template <int D>
struct Few {
  static constexpr int TILE = kTileBytes<D>, WAVE = 4 * TILE, ROWS_AT = kWaves * WAVE, STATS_AT = ROWS_AT + 2 * TILE;
  // two slots of keys and values a wave; Q, dO; -log2(e) lse, -delta, limits; sums of P dP a wave
  static constexpr int SUMS_AT = STATS_AT + 3 * 32 * 4, BYTES = SUMS_AT + kWaves * 32 * 4;
};

template <int D>
__global__ __launch_bounds__(kThreads) void k_bf16_dense_bwd_few(DenseBwd p) {
  constexpr int KS = D / 16, FT = D / 32, RB = 2 * D, PIECES = D / 8, TILE = kTileBytes<D>, LOADS = TILE / 1024;
  using L = Few<D>;
  auto swz = [](int row) { return D == 128 ? (row & 3) << 2 | ((row >> 2) & 3) : (row & 2) << 1 | ((row >> 2) & 3); };
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, hi = lane >> 5, c = lane & 31;
  const int parts = p.parts_q, unit = blockIdx.x, part = unit % parts, kh = unit / parts, b = kh / p.KH, hd = kh - b * p.KH;
  const int rows = p.group * p.Nq, keys = __builtin_amdgcn_readfirstlane(dense_seen_keys(p, b)), tiles = (p.Nkv + 31) >> 5;
  const int t0 = (int)((long long)tiles * part / parts), t1 = (int)((long long)tiles * (part + 1) / parts);
  const u16* Kp = (const u16*)p.K + b * p.k.batch + hd * p.k.head;
  const u16* Vp = (const u16*)p.V + b * p.v.batch + hd * p.v.head;
  const unsigned krow = (unsigned)p.k.token * 2u, vrow = (unsigned)p.v.token * 2u, lds0 = (unsigned)(unsigned long long)(const lds_void*)bwd_lds;
  const int mine = wave * L::WAVE;      // this wave's part of LDS

  // (keys that nothing sees are zeros)
  auto fetch = [&](int tile, int slot) {
    const int left = tile < t1 ? keys - 32 * tile : 0;
    const unsigned n = left <= 0 ? 0 : left < 32 ? left : 32;
    const u32x4 rk = rows_at(Kp + (long long)32 * tile * p.k.token, n ? (n - 1) * krow + RB : 0);
    const u32x4 rv = rows_at(Vp + (long long)32 * tile * p.v.token, n ? (n - 1) * vrow + RB : 0);
    const unsigned at = __builtin_amdgcn_readfirstlane(lds0 + mine + slot * 2 * TILE);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int s = j * 64 + lane, row = s / PIECES, piece = (s % PIECES) ^ swz(row);
      load_lds_16B(rk, at + j * 1024, row * krow + piece * 16);
      load_lds_16B(rv, at + TILE + j * 1024, row * vrow + piece * 16);
    }
  };
  fetch(t0 + wave, 0);

  // the rows: row r is query r % Nq of head r / Nq of those that share the keys
  int* const lims = (int*)(bwd_lds + L::STATS_AT) + 64;
  float* const stats = (float*)(bwd_lds + L::STATS_AT);
  {
    constexpr int PER = 32 * PIECES / kThreads;         // pieces of an array a thread moves, all of one row
    const int r = tid / (PIECES / PER), piece0 = tid % (PIECES / PER) * PER;
    const bool in = r < rows;
    const int gh = in ? r / p.Nq : 0, q = in ? r - gh * p.Nq : 0, hq = hd * p.group + gh;
    const u16* Qp = (const u16*)p.Q + b * p.q.batch + hq * p.q.head + q * p.q.token;
    const u16* dOp = (const u16*)p.dO + b * p.dout.batch + hq * p.dout.head + q * p.dout.token;
    const u16* Op = (const u16*)p.O + b * p.o.batch + hq * p.o.head + q * p.o.token;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int piece = piece0 + j;
      bf16x8 x = ld_global_16B(Qp + 8 * piece), y = ld_global_16B(dOp + 8 * piece);
      const bf16x8 o = ld_global_16B(Op + 8 * piece);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf((float)o[e], (float)y[e], sum);
      if (!in) x = y = bf16x8{};
      char* to = bwd_lds + L::ROWS_AT + r * RB + (piece ^ swz(r)) * 16;
      *(bf16x8*)to = x;
      *(bf16x8*)(to + TILE) = y;
    }
    sum = row8_sum(sum);                                 // (eight threads to a row)
    static_assert(PIECES / PER == 8, "");
    if ((tid & 7) == 0) {
      const float l = p.lse[((long long)b * p.H + hq) * p.Nq + q];
      stats[r] = !in || l == -INFINITY ? -INFINITY : -kLog2e * l;
      stats[32 + r] = in ? -sum : 0.f;
      lims[r] = in ? dense_last_key(p, q, keys) : 0;
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  const float scale2 = p.scale * kLog2e, nlq = stats[c];
  const int limq = lims[c], free_keys = dense_last_key(p, 0, keys);     // (the limits rise with the query)
  const int row_at = c * RB + (swz(c) ^ hi) * 16;
  auto row_op = [&](int at, int ks) { return *(const bf16x8*)(bwd_lds + at + (row_at ^ (32 * ks))); };
  // a sequence of few keys in a tensor of many: delta is the sum of P dP, as in k_bf16_dense_bwd_stats (a run of keys that
  // the sequence has none of needs no delta)
  if (keys <= kFewKeys && 32 * t0 < keys) {
    const int k0 = 32 * wave;
    const long long kr = k0 + c < keys ? k0 + c : keys - 1;
    const u16 *Kr = Kp + kr * p.k.token + 8 * hi, *Vr = Vp + kr * p.v.token + 8 * hi;
    f32x16 sv = {}, dp = {};         // rows: keys, columns: queries
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sv = mfma32(ld_global_16B(Kr + 16 * ks), row_op(L::ROWS_AT, ks), sv);
      dp = mfma32(ld_global_16B(Vr + 16 * ks), row_op(L::ROWS_AT + TILE, ks), dp);
    }
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float x = exp2_fast(fmaf(sv[r], scale2, nlq)) * dp[r];
      sum += k0 + 8 * (r >> 2) + 4 * hi + (r & 3) < limq ? x : 0.f;
    }
    sum += __shfl_xor(sum, 32);
    float* sums = (float*)(bwd_lds + L::SUMS_AT);
    if (hi == 0) sums[wave * 32 + c] = sum;
    __syncthreads();
    if (tid < 32) stats[32 + c] = -((sums[c] + sums[32 + c]) + (sums[64 + c] + sums[96 + c]));
    __syncthreads();
  }
  fetch(t0 + wave + kWaves, 1);

  const float ndq = stats[32 + c];
  const int G = lane >> 4, s = lane & 15, trow = 4 * hi + (s >> 2);
  const int tr_at = trow * RB + ((2 * (G & 1) + ((s >> 1) & 1)) ^ swz(trow)) * 16 + 8 * (s & 1);
  auto tr_op = [&](int at, int f, int kk) {
    const char* lo = bwd_lds + at + (tr_at ^ (64 * f)) + 16 * kk * RB;
    const char* up = bwd_lds + at + (tr_at ^ (64 * f + 32)) + (16 * kk + 8) * RB;
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(ld_lds_tr((const u16*)lo), ld_lds_tr((const u16*)up), 0, 1, 2, 3, 4, 5, 6, 7));
  };
  f32x16 dq[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) dq[f] = f32x16{};

  for (int tile = t0 + wave, slot = 0; tile < t1; tile += kWaves, slot ^= 1) {
    const int kt = mine + slot * 2 * TILE, vt = kt + TILE, key0 = 32 * tile, key = key0 + c;
    const bool edge = key0 + 32 > free_keys;
    f32x16 sv = {}, dp, st = {}, dt;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 x = *(const f32x4*)(stats + 32 + 8 * j + 4 * hi);
#pragma unroll
      for (int r = 0; r < 4; ++r) { dp[4 * j + r] = x[r]; dt[4 * j + r] = ndq; }
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 k = row_op(kt, ks), v = row_op(vt, ks), q = row_op(L::ROWS_AT, ks), d = row_op(L::ROWS_AT + TILE, ks);
      sv = mfma32(q, k, sv);
      dp = mfma32(d, v, dp);
      st = mfma32(k, q, st);
      dt = mfma32(v, d, dt);
    }
    bf16x8 pb[2], db[2], dbt[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 nl = *(const f32x4*)(stats + 8 * j + 4 * hi);
      const int* lr = lims + 8 * j + 4 * hi;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = 4 * j + r;
        float w = exp2_fast(fmaf(sv[e], scale2, nl[r])), wt = exp2_fast(fmaf(st[e], scale2, nlq));
        float d = w * dp[e], g = wt * dt[e];
        if (edge) {
          if (key >= lr[r]) w = d = 0.f;
          if (key0 + 8 * j + 4 * hi + r >= limq) g = 0.f;
        }
        pb[e >> 3][e & 7] = (__bf16)w;
        db[e >> 3][e & 7] = (__bf16)d;
        dbt[e >> 3][e & 7] = (__bf16)g;
      }
    }
    f32x16 dv[FT], dk[FT];
#pragma unroll
    for (int f = 0; f < FT; ++f) {
      dv[f] = dk[f] = f32x16{};
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        dv[f] = mfma32(tr_op(L::ROWS_AT + TILE, f, kk), pb[kk], dv[f]);
        dk[f] = mfma32(tr_op(L::ROWS_AT, f, kk), db[kk], dk[f]);
        dq[f] = mfma32(tr_op(kt, f, kk), dbt[kk], dq[f]);
      }
    }
    // dK in the place of K, dV in that of V, then row by row to memory
    const bool live = key < keys;
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        char* to = bwd_lds + c * RB + (((4 * f + j) ^ swz(c)) * 16) + 8 * hi;
        f32x4 x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = live ? dk[f][4 * j + e] * p.scale : 0.f;
          y[e] = live ? dv[f][4 * j + e] : 0.f;
        }
        *(bf16x4*)(to + kt) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
        *(bf16x4*)(to + vt) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
      }
    u32x4 ok[LOADS], ov[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      ok[j] = *(const u32x4*)(bwd_lds + kt + j * 1024 + lane * 16);
      ov[j] = *(const u32x4*)(bwd_lds + vt + j * 1024 + lane * 16);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");    // the next tile is here, and the last one's rows are written
    u16* tk = (u16*)p.dK + b * p.dk.batch + hd * p.dk.head;
    u16* tv = (u16*)p.dV + b * p.dv.batch + hd * p.dv.head;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int q = j * 64 + lane, row = q / PIECES, piece = (q % PIECES) ^ swz(row);
      const long long r = key0 + row;
      if (r < p.Nkv) {
        *(u32x4*)(tk + r * p.dk.token + 8 * piece) = ok[j];
        *(u32x4*)(tv + r * p.dv.token + 8 * piece) = ov[j];
      }
    }
    fetch(tile + 2 * kWaves, slot);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing is on its way to LDS
  __syncthreads();
  // dQ over the waves: [wave][row][D + 4] floats
  constexpr int LD = D + 4;
  static_assert(kWaves * 32 * LD * 4 <= L::ROWS_AT, "fits the tiles' place");
  float* sums = (float*)bwd_lds;
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(f32x4*)(sums + (wave * 32 + c) * LD + 32 * f + 8 * j + 4 * hi) = f32x4{dq[f][4 * j], dq[f][4 * j + 1], dq[f][4 * j + 2], dq[f][4 * j + 3]};
  __syncthreads();
  for (int i = tid; i < rows * (D / 4); i += kThreads) {
    const int r = i / (D / 4), f = 4 * (i % (D / 4)), gh = r / p.Nq;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x = x + *(const f32x4*)(sums + (w * 32 + r) * LD + f);
    const long long bh = (long long)b * p.H + hd * p.group + gh;
    *(f32x4*)(p.pq + (((long long)part * p.B * p.H + bh) * p.Nq + (r - gh * p.Nq)) * D + f) = x * p.scale;
  }
}

// (Where the tensor has a few keys, what memory costs does not matter.)
bool few_queries(const DenseBwd& p) { return (long long)p.group * p.Nq <= 32 && dense_last_key(p, 0, p.Nkv) > kFewKeys; }

template <int D>
hipError_t run(const DenseBwd& p, hipStream_t s) {
  hipError_t e;
  if (few_queries(p)) {
    constexpr int lds = Few<D>::BYTES;
    e = hipFuncSetAttribute((const void*)k_bf16_dense_bwd_few<D>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    k_bf16_dense_bwd_few<D><<<(unsigned)(p.B * p.KH * p.parts_q), kThreads, lds, s>>>(p);
    e = hipGetLastError();
    return e != hipSuccess ? e : launch_dense_bwd_join(p, true, false, MRT_BF16, s);
  }
  constexpr int lds = Stream<D, true>::RING;
  static_assert(lds >= Stream<D, false>::RING, "the ring of either");
  const int nqb = (p.Nq + 31) / 32;
  k_bf16_dense_bwd_stats<D><<<(unsigned)(p.B * p.H) * nqb, kThreads, 0, s>>>(p, nqb);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long keys = (p.Nkv + kRows - 1) / kRows * (long long)(p.B * p.KH) * p.parts_kv;
  const long long queries = (p.Nq + kRows - 1) / kRows * (long long)(p.B * p.H) * p.parts_q;
  const bool pq = p.parts_q > 1, pkv = p.parts_kv > 1;
  const auto kernel = pq ? pkv ? k_bf16_dense_bwd<D, true, true> : k_bf16_dense_bwd<D, true, false>
                         : pkv ? k_bf16_dense_bwd<D, false, true> : k_bf16_dense_bwd<D, false, false>;
  e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  kernel<<<(unsigned)(keys + queries), kThreads, lds, s>>>(p, (int)keys);
  e = hipGetLastError();
  return e != hipSuccess || !(pq || pkv) ? e : launch_dense_bwd_join(p, pq, pkv, MRT_BF16, s);
}

}  // namespace

DenseBwdShape bf16_dense_bwd_shape(const DenseBwd& p) {
  if (!few_queries(p)) return dense_bwd_shape(p, kRows, kStep, p.d == 64 ? 0.57 : 0.80, p.d == 64 ? 0.59 : 1.08);
  // few queries: runs of key tiles that fill the chip in whole rounds (a round costs a workgroup as much as half a tile)
  const long long cus = compute_units(), heads = (long long)p.B * p.KH, tiles = (p.Nkv + 31) / 32;
  double least = INFINITY;
  int best = 1;
  for (int parts = 1; parts <= 64 && parts <= tiles; ++parts) {
    const double cost = (double)((heads * parts + cus - 1) / cus) * ((double)((tiles + 4 * parts - 1) / (4 * parts)) + 0.5);
    if (cost < least) { least = cost; best = parts; }
  }
  return {best, 1, true, false};
}

hipError_t launch_bf16_dense_bwd(const DenseBwd& p, hipStream_t s) { return p.d == 64 ? run<64>(p, s) : run<128>(p, s); }

}  // namespace mrt
