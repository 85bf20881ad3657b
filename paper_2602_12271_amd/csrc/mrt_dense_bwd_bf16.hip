// Backward pass of the dense softmax attention on the bf16 matrix unit.
#include "mrt_dense_train.hpp"
#include "mrt_bf16_tiles.hpp"

#include <algorithm>

namespace mrt {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((address_space(3))) void lds_void;

__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// global memory (zeros beyond the resource's end) -> LDS: lane i's bytes to at + SIZE i
__device__ inline void load_lds_16B(__amdgpu_buffer_rsrc_t r, char* at, unsigned voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)at, 16, voff, 0, 0, 0);
}
__device__ inline void load_lds_4B(__amdgpu_buffer_rsrc_t r, char* at, unsigned voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)at, 4, voff, 0, 0, 0);
}
// waits for this wave's loads but the last N, and for its LDS reads, then for the other waves
template <int N> __device__ inline void wait_and_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

constexpr int kStep = 32;      // streamed rows a step
constexpr int kSlots = 4;      // LDS ring of steps: one is consumed, three are on their way

// LDS tile of 32 rows of D bf16, not padded (loads write LDS directly, 64 consecutive 16-byte pieces an
// instruction): piece p of row r lies at p ^ swz(r).
template <int D> __device__ inline int swz(int row) { return D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; }
template <int D> constexpr int kTileBytes = kStep * D * 2;
template <int D, bool KV> constexpr int kSlotBytes = 2 * kTileBytes<D> + (KV ? 256 : 0);
template <int D, bool KV> constexpr int kBwdLds = kSlots * kSlotBytes<D, KV>;

__device__ inline float half_sum(float x) {      // over the two lanes that share lane % 32
  float a = x, b = x;
  row_swap32(a, b);
  return a + b;
}

// One workgroup owns 32 NT W rows of one (batch, head): keys (KV) or queries; every wave 32 NT of them, whose
// operands and gradients stay in its registers.  The rows of the other side stream through LDS, 32 a step.
template <int D, int NT, int W, bool KV, bool PART>
__global__ __launch_bounds__(64 * W) void k_bf16_dense_bwd(DenseBwd p) {
  constexpr int KS = D / 16, FT = D / 32, ROWS = 32 * NT * W, RB = 2 * D, PIECES = D / 8;
  constexpr int TILE_LOADS = kTileBytes<D> / 1024, LOADS = 2 * TILE_LOADS / W;   // of one array's tile; of a wave's share of both
  constexpr int PERSTEP = LOADS + (KV ? 1 : 0);
  static_assert(LOADS * W == 2 * TILE_LOADS && (TILE_LOADS % W == 0 || W % TILE_LOADS == 0), "whole loads, of one array each");
  extern __shared__ __attribute__((aligned(1024))) char bwd_lds[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, hi = lane >> 5, c = lane & 31;

  const int n_own = KV ? p.Nkv : p.Nq, n_heads = p.B * (KV ? p.KH : p.H);
  const int tiles = (n_own + ROWS - 1) / ROWS, parts = PART ? (KV ? p.parts_kv : p.parts_q) : 1;
  int unit = blockIdx.x;
  const int total = gridDim.x;
  int bh, tile, part = 0;
  if (p.cc == 0) {
    const int xcd = unit & 7;
    unit = xcd * (total >> 3) + (xcd < (total & 7) ? xcd : (total & 7)) + (unit >> 3);
    tile = unit % tiles;
    unit /= tiles;
    part = unit % parts;
    bh = unit / parts;
  } else {
    bh = unit % n_heads;
    unit /= n_heads;
    part = unit % parts;
    tile = unit / parts;
    if (!KV) tile = tiles - 1 - tile;
  }
  const int b = bh / (KV ? p.KH : p.H), hd = bh - b * (KV ? p.KH : p.H), kvh = KV ? hd : hd / p.group;
  const int own0 = tile * ROWS, keys = dense_keys(p, b);
  const int own_last = own0 + ROWS < n_own ? own0 + ROWS - 1 : n_own - 1;

  // the streamed rows: queries qfirst .. Nq of every head that shares these keys, or keys 0 .. klast
  const int qfirst = KV ? dense_first_query(p, own0) & ~31 : 0;
  const int s_end = KV ? p.Nq : dense_last_key(p, own_last, keys);
  const int per_head = KV ? (own0 < keys ? (s_end - qfirst + 31) >> 5 : 0) : (s_end + 31) >> 5;
  const int all = KV ? per_head * p.group : per_head;
  const int i0 = PART ? (int)((long long)all * part / parts) : 0, i1 = PART ? (int)((long long)all * (part + 1) / parts) : all;

  const u16* own_a = KV ? (const u16*)p.K + b * p.k.batch + hd * p.k.head : (const u16*)p.Q + b * p.q.batch + hd * p.q.head;
  const u16* own_b = KV ? (const u16*)p.V + b * p.v.batch + hd * p.v.head : (const u16*)p.dO + b * p.dout.batch + hd * p.dout.head;
  const long long own_at = KV ? p.k.token : p.q.token, own_bt = KV ? p.v.token : p.dout.token;
  const u16* st_a = KV ? (const u16*)p.Q + b * p.q.batch + (long long)hd * p.group * p.q.head
                       : (const u16*)p.K + b * p.k.batch + kvh * p.k.head;
  const u16* st_b = KV ? (const u16*)p.dO + b * p.dout.batch + (long long)hd * p.group * p.dout.head
                       : (const u16*)p.V + b * p.v.batch + kvh * p.v.head;
  const long long st_at = KV ? p.q.token : p.k.token, st_bt = KV ? p.dout.token : p.v.token;
  const int nqb = (p.Nq + 31) >> 5;

  // streamed tile -> LDS
  const unsigned arow = (unsigned)st_at * 2u, brow = (unsigned)st_bt * 2u;
  unsigned voff[LOADS];
  auto of_b = [&](int j) { return TILE_LOADS % W == 0 ? j * W >= TILE_LOADS : wave >= TILE_LOADS; };   // load j is of the second array
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int s = (j * W + wave) % TILE_LOADS * 64 + lane, row = s / PIECES, piece = (s % PIECES) ^ swz<D>(row);
    voff[j] = row * (of_b(j) ? brow : arow) + piece * 16;
  }
  auto issue = [&](int i) {
    const int slot = (i & (kSlots - 1)) * kSlotBytes<D, KV>;
    int gh = 0, row = i << 5;
    if (KV) {
      gh = p.group == 1 ? 0 : i / (per_head > 0 ? per_head : 1);
      row = qfirst + ((i - gh * per_head) << 5);
    }
    const int left = i < i1 ? s_end - row : 0;
    const unsigned rows = left < 32 ? left : 32;
    const u16* a = st_a + (KV ? gh * p.q.head : 0) + row * st_at;
    const u16* bb = st_b + (KV ? gh * p.dout.head : 0) + row * st_bt;
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void*)a, 0, rows ? (rows - 1) * arow + RB : 0, 0x00020000);
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc((void*)bb, 0, rows ? (rows - 1) * brow + RB : 0, 0x00020000);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) load_lds_16B(of_b(j) ? rb : ra, bwd_lds + slot + (j * W + wave) * 1024, voff[j]);
    if constexpr (KV) {       // (every wave writes the same 256 bytes: all wait for the same number of loads)
      const float* st = p.stats + ((long long)(b * p.H + hd * p.group + gh) * nqb + (row >> 5)) * 64;
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)st, 0, rows ? 256 : 0, 0x00020000);
      load_lds_4B(rs, bwd_lds + slot + 2 * kTileBytes<D>, lane * 4);
    }
  };
  issue(i0);
  issue(i0 + 1);
  issue(i0 + 2);

  // operands of this wave's rows
  const int ow0 = own0 + 32 * NT * wave;
  bf16x8 oa[NT][KS], ob[NT][KS];
  int lim[NT];                         // KV: first query that sees the lane's key; else: its query's number of keys
  float nlse[NT], ndelta[NT];          // (queries) -log2(e) lse, -delta
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = ow0 + 32 * t + c, rc = r < n_own ? r : n_own - 1;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      oa[t][ks] = ld_global_16B(own_a + rc * own_at + 16 * ks + 8 * hi);
      ob[t][ks] = ld_global_16B(own_b + rc * own_bt + 16 * ks + 8 * hi);
    }
    lim[t] = KV ? dense_first_query(p, rc) : dense_last_key(p, rc, keys);
    if constexpr (!KV) {
      const u16* orow = (const u16*)p.O + b * p.o.batch + hd * p.o.head + rc * p.o.token;
      float sum = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 o = ld_global_16B(orow + 16 * ks + 8 * hi);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf((float)o[e], (float)ob[t][ks][e], sum);
      }
      ndelta[t] = -half_sum(sum);
      const float l = p.lse[(long long)bh * p.Nq + rc];
      const bool none = l == -INFINITY;
      nlse[t] = none ? -INFINITY : -kLog2e * l;
      if (part == 0 && hi == 0 && r < nqb * 32) {
        float* st = p.stats + ((long long)bh * nqb + (r >> 5)) * 64 + (r & 31);
        st[0] = none || r >= p.Nq ? -INFINITY : -l / p.scale;
        st[32] = r >= p.Nq ? 0.f : ndelta[t];
      }
    }
  }
  const float scale2 = p.scale * kLog2e;
  f32x16 g1[KV ? NT : 1][FT], g2[NT][FT];    // dV^T; dK^T or dQ^T
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (KV) g1[t][f][r] = 0.f;
        g2[t][f][r] = 0.f;
      }

  // where a lane reads its operands of a tile
  int arow_at[KS], tr_at[FT];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) arow_at[ks] = c * RB + ((2 * ks) ^ swz<D>(c)) * 16 + hi * 16;
  const int G = lane >> 4, s = lane & 15, trow = 4 * hi + (s >> 2);
#pragma unroll
  for (int f = 0; f < FT; ++f)       // (rows 8 apart are swizzled alike)
    tr_at[f] = trow * RB + (((4 * f + 2 * (G & 1)) ^ swz<D>(trow)) * 16) + 8 * (s & 3);

  auto row_op = [&](const char* at, int ks) { return *(const bf16x8*)(at + arow_at[ks]); };
  auto tr_op = [&](const char* at, int f, int kk) {
    const u16* q = (const u16*)(at + tr_at[f] + 16 * kk * RB);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(ld_lds_tr(q), ld_lds_tr(q + 8 * D), 0, 1, 2, 3, 4, 5, 6, 7));
  };

  for (int i = i0; i < i1; ++i) {
    wait_and_meet<2 * PERSTEP>();
    issue(i + 3);
    const char* at = bwd_lds + (i & (kSlots - 1)) * kSlotBytes<D, KV>;
    const char* bt = at + kTileBytes<D>;
    int row = i << 5;
    if (KV) row = qfirst + ((p.group == 1 ? i : i % per_head) << 5);

    f32x16 sv[NT], dp[NT];
    if constexpr (KV) {
      const float* st = (const float*)(bt + kTileBytes<D>) + 4 * hi;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 l = *(const f32x4*)(st + 8 * j), dl = *(const f32x4*)(st + 32 + 8 * j);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) { sv[t][4 * j + r] = l[r]; dp[t][4 * j + r] = dl[r]; }
      }
    } else {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) { sv[t][r] = 0.f; dp[t][r] = ndelta[t]; }
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 a = row_op(at, ks);
#pragma unroll
      for (int t = 0; t < NT; ++t) sv[t] = mfma32(a, oa[t][ks], sv[t]);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 a = row_op(bt, ks);
#pragma unroll
      for (int t = 0; t < NT; ++t) dp[t] = mfma32(a, ob[t][ks], dp[t]);
    }
    // a step that some row of the workgroup does not see whole
    const bool edge = KV ? p.cc != 0 && row < dense_first_query(p, own_last) : row + 32 > dense_last_key(p, own0, keys);
    if (edge) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int at_row = row + 8 * (r >> 2) + 4 * hi + (r & 3);
          if (KV ? at_row < lim[t] : at_row >= lim[t]) { sv[t][r] = -INFINITY; dp[t][r] = 0.f; }
        }
    }
    bf16x8 pb[NT][2], db[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = exp2_fast(KV ? sv[t][r] * scale2 : fmaf(sv[t][r], scale2, nlse[t]));
        const float d = w * dp[t][r];
        pb[t][r >> 3][r & 7] = (__bf16)w;
        db[t][r >> 3][r & 7] = (__bf16)d;
      }
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        if constexpr (KV) {
          const bf16x8 a = tr_op(bt, f, kk);
#pragma unroll
          for (int t = 0; t < NT; ++t) g1[t][f] = mfma32(a, pb[t][kk], g1[t][f]);
        }
      }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        const bf16x8 a = tr_op(at, f, kk);
#pragma unroll
        for (int t = 0; t < NT; ++t) g2[t][f] = mfma32(a, db[t][kk], g2[t][f]);
      }
  }

  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing is on its way to LDS when the workgroup leaves it

  typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = ow0 + 32 * t + c;
    if (r >= n_own) continue;
    const bool live = KV ? r < keys : true;
    if constexpr (PART) {
      float* to = (KV ? p.pk : p.pq) + (((long long)part * n_heads + bh) * n_own + r) * D + 4 * hi;
      float* tv = KV ? p.pv + (((long long)part * n_heads + bh) * n_own + r) * D + 4 * hi : nullptr;
#pragma unroll
      for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f32x4 x, y;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = live ? g2[t][f][4 * j + e] * p.scale : 0.f;
            if constexpr (KV) y[e] = live ? g1[t][f][4 * j + e] : 0.f;
          }
          *(f32x4*)(to + 32 * f + 8 * j) = x;
          if constexpr (KV) *(f32x4*)(tv + 32 * f + 8 * j) = y;
        }
    } else {
      u16* to = (KV ? (u16*)p.dK + b * p.dk.batch + hd * p.dk.head + r * p.dk.token
                    : (u16*)p.dQ + b * p.dq.batch + hd * p.dq.head + r * p.dq.token) + 4 * hi;
      u16* tv = KV ? (u16*)p.dV + b * p.dv.batch + hd * p.dv.head + r * p.dv.token + 4 * hi : nullptr;
#pragma unroll
      for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bf16x4 x, y;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = (__bf16)(live ? g2[t][f][4 * j + e] * p.scale : 0.f);
            if constexpr (KV) y[e] = (__bf16)(live ? g1[t][f][4 * j + e] : 0.f);
          }
          *(bf16x4*)(to + 32 * f + 8 * j) = x;
          if constexpr (KV) *(bf16x4*)(tv + 32 * f + 8 * j) = y;
        }
    }
  }
}

template <int D, int NT, int W, bool KV, bool PART>
hipError_t run_bwd(const DenseBwd& p, hipStream_t s) {
  constexpr int lds = kBwdLds<D, KV>, rows = 32 * NT * W;
  const hipError_t e = hipFuncSetAttribute((const void*)k_bf16_dense_bwd<D, NT, W, KV, PART>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  const int n = KV ? p.Nkv : p.Nq, heads = p.B * (KV ? p.KH : p.H), parts = PART ? (KV ? p.parts_kv : p.parts_q) : 1;
  k_bf16_dense_bwd<D, NT, W, KV, PART><<<(n + rows - 1) / rows * heads * parts, 64 * W, lds, s>>>(p);
  return hipGetLastError();
}

template <int D, int NT, int W, bool KV>
hipError_t run_parts(const DenseBwd& p, hipStream_t s) {
  if ((KV ? p.parts_kv : p.parts_q) == 1) return run_bwd<D, NT, W, KV, false>(p, s);
  const hipError_t e = run_bwd<D, NT, W, KV, true>(p, s);
  return e != hipSuccess ? e : launch_dense_bwd_join(p, KV, MRT_BF16, s);
}

}  // namespace

DenseBwdShape bf16_dense_bwd_shape(const DenseBwd& p) {
  DenseBwdShape shape = {256, 1, p.d == 64 ? 256 : 128, 1};
  const long long cus = compute_units(), most = 1 << 27;      // elements of the parts
  auto parts = [&](long long rows, long long heads, long long tile, long long streamed) {
    const long long wgs = (rows + tile - 1) / tile * heads, steps = (streamed + 31) / 32;
    long long n = wgs < cus ? cus / wgs : 1;
    if (n > steps / 4) n = steps / 4;
    if (n > most / (rows * heads * p.d)) n = most / (rows * heads * p.d);
    return (int)(n < 1 ? 1 : n);
  };
  shape.parts_q = parts(p.Nq, (long long)p.B * p.H, shape.rows_q, p.Nkv);
  shape.parts_kv = parts(p.Nkv, (long long)p.B * p.KH, shape.rows_kv, (long long)p.Nq * p.group);
  return shape;
}

hipError_t launch_bf16_dense_bwd(const DenseBwd& p, const DenseBwdShape& shape, hipStream_t s) {
  (void)shape;
  hipError_t e;
  if (p.d == 64) {
    e = run_parts<64, 2, 4, false>(p, s);
    return e != hipSuccess ? e : run_parts<64, 1, 8, true>(p, s);
  }
  e = run_parts<128, 2, 4, false>(p, s);
  return e != hipSuccess ? e : run_parts<128, 1, 4, true>(p, s);
}

#ifdef PROBE
hipError_t (*probes[])(const DenseBwd&, hipStream_t) = {PROBE};
#endif
}  // namespace mrt
