// The kernels of the dense softmax attention on the bf16 matrix unit (Sec. 2.2), chunk-causal by token: keys and values
// in bf16 (mrt_dense_bf16.hip) or in a cache of 8 bits (mrt_dense_cache8.hip).
// See the head of mrt_bf16.hip for the register layouts.
//
// Eight waves, two to a SIMD, each owning QT query tiles of 16.  A step of 64 keys is a vector phase
// (maxima, exponentials, packing, the refill of the LDS ring) and a matrix phase (first product of the
// next step, second product of this one, their LDS reads), and the two halves of the workgroup run one
// phase apart: one wave of a SIMD feeds the matrix unit while the other one has the vector ALU.  The
// barrier that ends every phase keeps them so.  (Without it the waves drift into step and the two
// units take turns: a matrix unit busy 35 % of the time.)  What bounds the kernel then is the vector
// phase (vector instructions issue at half rate under the other wave's products) and about 150 clocks
// of barrier per phase; hence phases of 64 keys (two chunks).  The sums of the probabilities are fp32
// additions of the unrounded values: a product with ones over the rounded ones takes them off the
// vector ALU (3 to 6 % of a call), but shortens the denominator by up to 2^-8 where the roundings agree.
//
// LDS rows are padded to D + 16 elements (288 bytes at D = 128): the 16-byte key reads and the
// transposed value reads of 16 contiguous features then both run free of bank conflicts (4.0 and 2.8
// clocks per wave instruction and CU measured; a 16-byte XOR swizzle 6.0 and 4.0).
//
// WK = 1: every wave sees all keys.  WK = 2: waves w and w + 4 share their queries and take one half of
// every 64 keys (half the queries per workgroup, so twice the workgroups); the halves are merged at the
// end.
//
// PART: a workgroup takes one of `parts` runs of 64-key pairs and leaves its accumulators, references and
// sums in fp32 for k_dense_merge; for calls of few queries (dense_shape).
#pragma once
#include "mrt_internal.hpp"
#include "mrt_bf16_tiles.hpp"
#include "mrt_cache8.hpp"

namespace mrt {

struct DenseShape {
  int queries, parts;    // queries per workgroup, workgroups that share the keys of one query tile
};

namespace {

// A query's softmax reference is raised only when a logit exceeds it by more than this (base 2):
// every probability is then at most 2^kGrow, and the ratio sum(p v) / sum(p) does not depend on it.
constexpr float kGrow = 8.0f;
constexpr float kNoKey = -__FLT_MAX__;   // reference of a query that has seen no key
// Beyond this the rounding of a reference, which its own logit's exponent would contain (one fma), is no
// longer small beside kGrow: every step then counts as one that raises it, and there the exponents are
// formed from logits that are rounded first.  (A choice between the two on the common path costs a
// quarter of the call at 64 features: it parts the exponentials from the rest of the vector phase.)
constexpr float kFarRef = 0x1p20f;
constexpr int kDenseWaves = 8, kDenseThreads = 64 * kDenseWaves;
// LDS ring of 64-key pairs of chunks: while pair i is consumed, pair i + 1 is resident, pair i + 2 is
// being written and pair i + 3 is in flight from global memory.
constexpr int kDenseSlots = 4;
constexpr int kAhead = 5;    // operand reads ahead of their products (3, 5 and 7 measured alike)
template <int D> constexpr int kDenseLd = D + 16;                          // elements per LDS row
template <int D> constexpr int kDenseSlot = 2 * 64 * kDenseLd<D>;          // 64 keys, then 64 values
template <int D> constexpr size_t kDenseLds = (size_t)kDenseSlots * kDenseSlot<D> * 2;

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;

// 64 rows of D bf16 between global memory and LDS.  Buffer loads return zeros beyond the last row, so
// no load is clamped or conditional.
template <int D>
struct DenseTile {
  static constexpr int CPR = D / 8, N = 64 * CPR / kDenseThreads, RSTEP = kDenseThreads / CPR;
  u32x4 v[N];
  // at: byte offset of the tile's first row
  __device__ inline void load(__amdgpu_buffer_rsrc_t rsrc, unsigned voff, unsigned at, unsigned rowbytes) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      v[i] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff + (at + (unsigned)(i * RSTEP) * rowbytes), 0, 0);
  }
  __device__ inline void store(u16* dst, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i) *(u32x4*)(dst + (tid / CPR + i * RSTEP) * kDenseLd<D> + 8 * (tid % CPR)) = v[i];
  }
};

// 64 rows of D codes of an 8-bit cache between global memory and LDS, where they are bf16: a code times its block's power
// of two is a bf16 number exactly, so that everything behind the ring is the kernel of bf16 keys and values.  A thread owns
// 8 codes, which are 16 contiguous bytes in LDS, and fetches their exponent with them (e4m3: one instruction for two
// values, scaled; whole numbers: 2.5 a value).
template <int D, bool E4M3>
struct DenseTile8 {
  static constexpr int CPR = D / 8, N = 64 * CPR / kDenseThreads, RSTEP = kDenseThreads / CPR;
  u32x2 v[N];
  unsigned char e[N];
  // MOVES: the resource begins at the tile's first row, so that the vector ALU, which bounds the kernel, forms no addresses
  // (e4m3, 128 features, 12 heads of 4680 queries of 32760 keys 848 -> 835 us; whole numbers 968 -> 996, 64 features the same)
  static constexpr bool MOVES = E4M3 && D == 128;
  // key: the tile's first row, of which this thread has `row`; shift: log2 of the rows that share an exponent
  __device__ inline void load(__amdgpu_buffer_rsrc_t codes, unsigned voff, unsigned rowbytes, __amdgpu_buffer_rsrc_t exps, unsigned key,
                              unsigned row, int shift) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = __builtin_amdgcn_raw_buffer_load_b64(codes, voff + ((MOVES ? 0 : key) + (unsigned)(i * RSTEP)) * rowbytes, 0, 0);
      e[i] = __builtin_amdgcn_raw_buffer_load_b8(exps, (key + row + (unsigned)(i * RSTEP)) >> shift, 0, 0);
    }
  }
  __device__ inline void store(u16* dst, int tid) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float scale = cache8_scale(e[i]);
      *(bf16x8*)(dst + (tid / CPR + i * RSTEP) * kDenseLd<D> + 8 * (tid % CPR)) = cache8_values<E4M3>(v[i], scale);
    }
  }
};

// Keys query q sees: the frames up to the end of its own chunk, a prefix.
__host__ __device__ inline int dense_visible(const KParams& p, int q) {
  if (p.cc == 0) return p.Nkv;
  const long long lim = (long long)((p.qoff + q / p.hw) / p.cc + 1) * p.cc * p.hw;
  return lim < p.Nkv ? (int)lim : p.Nkv;
}

// Partial results of a call whose keys are split over `n` workgroups per query tile: every part's
// accumulators, softmax reference and sum of a query (row = (part, head, query)).
struct DenseParts {
  float* o;     // [part][bh][q][D]
  float2* ml;   // [part][bh][q]
  int n;
  unsigned heads;   // of the batch
  unsigned runs;    // heads x n where queries see different numbers of keys, else 0
};

template <typename Save> constexpr bool dense_codes = false;
template <bool E4M3> constexpr bool dense_codes<DenseCache8<E4M3>> = true;
template <int D, typename Save> struct DenseTileOf { using type = DenseTile<D>; };
template <int D, bool E4M3> struct DenseTileOf<D, DenseCache8<E4M3>> { using type = DenseTile8<D, E4M3>; };

// (64 features: two workgroups to a compute unit)
// Save = DenseSave: a training step's call (heads that share keys, sequences of their own lengths, row statistics);
// DenseCache8: the same over a cache of 8 bits
template <int D, int QT, int WK, bool PART, typename Save>
__global__ __launch_bounds__(kDenseThreads, D == 64 ? 4 : 2) void k_bf16_dense(KParams p, DenseParts parts, Save save) {
  constexpr bool SAVE = !std::is_same<Save, NoSave>::value, CODES = dense_codes<Save>;
  using Tile = typename DenseTileOf<D, Save>::type;
  constexpr int KS1 = D / 32, NVT = D / 16, LD = kDenseLd<D>, WQ = kDenseWaves / WK, WGQ = 16 * QT * WQ;
  constexpr int NS = 2 / WK, NT = 2 * NS;                 // 32-key chunks / 16-key tiles of a wave's step
  extern __shared__ __attribute__((aligned(16))) u16 dense_lds[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int wq = wave % WQ, wk = wave / WQ;
  const bool second = wave >= kDenseWaves / 2;           // the half that runs one phase behind
  auto visible = [&](int q) { return dense_visible(p, q); };
  // Workgroups reach the eight XCDs in turn: hand each XCD a contiguous run of (head, query tile)
  // units, so that the units that stream the same keys share its L2.  Under a mask that gives the query
  // tiles of a head different key counts the longest of all heads go first, or a long one is the last to
  // start (us, head by head | longest first, 128 features: 16 heads of 8192 causal tokens 452 | 271, 32 of
  // 4096 253 | 156, 12 of 14040 tokens in chunks of 4680 846 | 756, 32 of 2048 75 | 70; 64 features 549 | 465).
  // (The host says which, and how many heads there are: to find both out took a masked call of 7 us another 0.4.)
  const int nx = (p.Nq + WGQ - 1) / WGQ, total = gridDim.x, xcd = blockIdx.x & 7;
  int run, tile;                                                   // run = (head, part)
  if (parts.runs == 0) {
    const int unit = xcd * (total >> 3) + (xcd < (total & 7) ? xcd : (total & 7)) + (blockIdx.x >> 3);
    run = unit / nx;
    tile = unit - run * nx;
  } else {
    const unsigned round = blockIdx.x / parts.runs;
    tile = nx - 1 - (int)round;
    run = (int)(blockIdx.x - round * parts.runs);
  }
  int q0 = tile * WGQ;
  int bh = PART ? run / parts.n : run, part = PART ? run - bh * parts.n : 0;
  // CODES: of a call whose last round is shared (DenseRounds) the tile, counted from that round's first, or -1
  [[maybe_unused]] int rest = -1;
  [[maybe_unused]] bool own_rows = false;
  if constexpr (PART && CODES)
    if (save.rounds.rest > 0) {
      const DenseRounds& r = save.rounds;
      auto spread = [](int at, int n) { return (at & 7) * (n >> 3) + ((at & 7) < (n & 7) ? (at & 7) : (n & 7)) + (at >> 3); };
      int unit = blockIdx.x;
      if (unit < r.whole) unit = spread(unit, r.whole);
      else {
        const int x = spread(unit - r.whole, r.rest * parts.n);
        rest = x / parts.n;
        part = x - rest * parts.n;
        unit = r.whole + rest;
      }
      own_rows = rest < 0;
      bh = unit / nx;
      q0 = (unit - bh * nx) * WGQ;
    }
  // CODES, sequences of lengths of their own: the longest one's tiles go first, or they are the last to end, and every sequence's go to
  // all XCDs, each a run of them, or some have the longest one alone (us, as they come | so: 12 heads, 4680 queries of 14040, 9360,
  // 4680 and 0 keys 1485 | 766, of 14040 and 7000 739 | 567, of two times 32760 1698 | 1706; parted, 8 heads, 780 queries of 9360
  // and 300 84.7 | 82.0)
  if constexpr (CODES)
    if (save.by_length > 0) {
      const int units = nx * p.H * (PART ? parts.n : 1), rank = blockIdx.x / units, at = blockIdx.x - rank * units;
      const int len = lane < save.by_length ? min(max(save.kv_len[lane], 0), p.Nkv) : -1;
      int before = 0;
      for (int i = 0; i < save.by_length; ++i) {
        const int other = __builtin_amdgcn_readlane(len, i);
        before += other > len || (other == len && i < lane);
      }
      const int seq = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < save.by_length && before == rank));
      const int unit = (at & 7) * (units >> 3) + ((at & 7) < (units & 7) ? (at & 7) : (units & 7)) + (at >> 3);
      run = unit / nx;
      q0 = (unit - run * nx) * WGQ;
      const int head = PART ? run / parts.n : run;
      if constexpr (PART) part = run - head * parts.n;
      bh = seq * p.H + head;
    }
  const int b = bh / p.H, hd = bh - b * p.H;
  int kvh = hd;
  const int qw0 = q0 + 16 * QT * wq;                      // this wave's first query
  if constexpr (SAVE) {
    kvh = hd / save.group;
    if (save.kv_len) p.Nkv = __builtin_amdgcn_readfirstlane(min(max(save.kv_len[b], 0), p.Nkv));
    if (p.Nkv == 0) {                                     // an empty sequence
      long long row0 = PART ? ((long long)part * parts.heads + bh) * p.Nq : 0;
      if constexpr (PART && CODES)
        if (rest >= 0) row0 = ((long long)part * save.rounds.rest + rest) * WGQ - q0;
      for (int i = tid; i < WGQ * D; i += kDenseThreads) {
        const int q = q0 + i / D, f = i % D;
        if (q >= p.Nq) break;
        if (PART && !own_rows) {
          parts.o[(row0 + q) * D + f] = 0.f;
          if (f == 0) parts.ml[row0 + q] = make_float2(kNoKey, 0.f);
        } else {
          ((u16*)p.O)[b * p.os.batch + hd * p.os.head + (long long)q * p.os.token + f] = 0;
          if (f == 0) save.lse[(long long)bh * p.Nq + q] = -INFINITY;
        }
      }
      return;
    }
  }
  const int nkeys = visible(q0 + WGQ - 1 < p.Nq ? q0 + WGQ - 1 : p.Nq - 1), nfree = visible(q0);

  const u16* Qp = (const u16*)p.Q + b * p.qs.batch + hd * p.qs.head;
  bf16x8 qv[QT][KS1];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const int qi = qw0 + 16 * q + c, qc = qi < p.Nq ? qi : p.Nq - 1;
#pragma unroll
    for (int ks = 0; ks < KS1; ++ks) qv[q][ks] = ld_global_16B(Qp + (long long)qc * p.qs.token + 32 * ks + 8 * g);
  }

  using KV = typename std::conditional<CODES, unsigned char, u16>::type;
  constexpr unsigned EB = sizeof(KV);                     // bytes of a key's element
  const unsigned krow = (unsigned)p.ks.token * EB, vrow = (unsigned)p.vs.token * EB;     // bytes per token
  // 256 queries: the first half's 128 stop at key `mid`, and a pair of chunks ends there, so that no value
  // hidden from all of them meets their weights of zero (0 x inf); the rest is the second half's alone
  const int mid = WK == 1 ? visible(q0 + WGQ / 2 - 1 < p.Nq ? q0 + WGQ / 2 - 1 : p.Nq - 1) : nkeys;
  const int nmid = (mid + 63) >> 6, npairs = nmid + ((nkeys - mid + 63) >> 6);
  auto first_key = [&](int pr) { return pr < nmid ? 64 * pr : mid + 64 * (pr - nmid); };
  int p0 = PART ? part * npairs / parts.n : 0, p1 = PART ? (part + 1) * npairs / parts.n : npairs;   // this part's pairs
  if constexpr (PART && CODES)
    if (own_rows) p0 = 0, p1 = npairs;
  const KV* Kp = (const KV*)p.K + b * p.ks.batch + kvh * p.ks.head;
  const KV* Vp = (const KV*)p.V + b * p.vs.batch + kvh * p.vs.head;
  const unsigned kvoff = (unsigned)(tid / Tile::CPR) * krow + 8u * EB * (tid % Tile::CPR);
  const unsigned vvoff = (unsigned)(tid / Tile::CPR) * vrow + 8u * EB * (tid % Tile::CPR);
  Tile kt, vt;
  // (pairs past the end re-read the last one; nobody reads their slot, or only as masked keys)
  auto fetch = [&](int pr) {
    const int last = PART && p1 > p0 ? p1 : npairs, at = pr < last ? pr : last - 1, end = at < nmid ? mid : nkeys;
    const unsigned key = (unsigned)first_key(at), rows = (unsigned)(end - 1);
    if constexpr (CODES) {
      auto from = [&](const KV* base, unsigned row) {
        const unsigned first = Tile::MOVES ? key : 0;
        return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (unsigned)__builtin_amdgcn_readfirstlane(first * row)), 0,
                                                 __builtin_amdgcn_readfirstlane((rows - first) * row + D), 0x00020000);
      };
      const auto kr = from(Kp, krow), vr = from(Vp, vrow);
      const int last_exp = (int)(rows >> save.shift) + 1;
      const auto ke = __builtin_amdgcn_make_buffer_rsrc((void*)(save.k_exp + b * save.ke_batch + kvh * save.ke_head), 0, last_exp, 0x00020000);
      const auto ve = __builtin_amdgcn_make_buffer_rsrc((void*)(save.v_exp + b * save.ve_batch + kvh * save.ve_head), 0, last_exp, 0x00020000);
      kt.load(kr, kvoff, krow, ke, key, tid / Tile::CPR, save.shift);
      vt.load(vr, vvoff, vrow, ve, key, tid / Tile::CPR, save.shift);
    } else {
      kt.load(__builtin_amdgcn_make_buffer_rsrc((void*)Kp, 0, rows * krow + 2 * D, 0x00020000), kvoff, key * krow, krow);
      vt.load(__builtin_amdgcn_make_buffer_rsrc((void*)Vp, 0, rows * vrow + 2 * D, 0x00020000), vvoff, key * vrow, vrow);
    }
  };
  auto commit = [&](int slot) {
    u16* at = dense_lds + slot * kDenseSlot<D>;
    kt.store(at, tid);
    vt.store(at + 64 * LD, tid);
  };

  const float scale2 = p.scale * kLog2e;
  bf16x8 pb[QT][NS];
  f32x4 s[QT][NT], o[QT][NVT];
  float mref[QT], thr[QT];                // reference, the raw logit that would raise it (kFarRef: any would)
  float mul[QT], off[QT];                 // a step's exponents are s mul - off: scale and reference, or 1 and 0 (kFarRef)
  float lrun[QT];                         // this lane's sum of the (unrounded) probabilities
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    mref[q] = off[q] = kNoKey; mul[q] = scale2; thr[q] = -INFINITY; lrun[q] = 0.f;
#pragma unroll
    for (int vt = 0; vt < NVT; ++vt) o[q][vt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // A wave's keys of a pair start at row 32 wk (WK = 2) or 0.
  const int koff = (WK == 2 ? 32 * wk * LD : 0) + c * LD + 8 * g;
  const int voff = 64 * LD + (WK == 2 ? 32 * wk * LD : 0) + (4 * g + (c >> 2)) * LD + 4 * (c & 3);
  // The matrix phase: s = logits of the next step's keys (pair in kslot), o += the probabilities'
  // product with this step's values (pair in vslot).  Operands are read from LDS kAhead groups of
  // products ahead of their use, in this fixed order.
  constexpr int NK_OPS = NT * KS1, NV_OPS = NS * NVT, OPS = NK_OPS + NV_OPS;
  bf16x8 op[OPS];
  auto read_op = [&](int i, const u16* ka, const u16* va) {
    if (i < NK_OPS) {
      op[i] = ld_lds_16B(ka + 16 * (i % NT) * LD + 32 * (i / NT));
    } else {
      const u16* at = va + 32 * ((i - NK_OPS) / NVT) * LD + 16 * ((i - NK_OPS) % NVT);
      op[i] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(ld_lds_tr(at), ld_lds_tr(at + 16 * LD), 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  auto matrix = [&](int kslot, int vslot, bool with_v) {
    const u16* ka = dense_lds + kslot * kDenseSlot<D> + koff;
    const u16* va = dense_lds + vslot * kDenseSlot<D> + voff;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read_op(i, ka, va);
#pragma unroll
    for (int i = 0; i < OPS; ++i) {
      if (!with_v && i >= NK_OPS) break;
      if (i + kAhead < (with_v ? OPS : NK_OPS)) read_op(i + kAhead, ka, va);
      if (i < NK_OPS) {
#pragma unroll
        for (int q = 0; q < QT; ++q)
          s[q][i % NT] = mfma(op[i], qv[q][i / NT], i < NT ? f32x4{0.f, 0.f, 0.f, 0.f} : s[q][i % NT]);
      } else {
        const int st = (i - NK_OPS) / NVT, vt = (i - NK_OPS) % NVT;
#pragma unroll
        for (int q = 0; q < QT; ++q) o[q][vt] = mfma(op[i], pb[q][st], o[q][vt]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto top = [&](int q) {
    if constexpr (CODES) {                // (in an order that makes every instruction take two more)
      float m = s[q][0][0];
#pragma unroll
      for (int i = 1; i < 4 * NT; i += 2) m = i + 1 < 4 * NT ? fmaxf(fmaxf(m, s[q][i / 4][i % 4]), s[q][(i + 1) / 4][(i + 1) % 4]) : fmaxf(m, s[q][i / 4][i % 4]);
      return m;
    }
    float m = fmaxf(s[q][0][0], s[q][0][1]);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t > 0) m = fmaxf(m, fmaxf(s[q][t][0], s[q][t][1]));
      m = fmaxf(m, fmaxf(s[q][t][2], s[q][t][3]));
    }
    return m;
  };
  // the raw logits of the keys from c0 on are complete: mask them where they reach beyond a query's
  // keys or the pair's end, raise the references they exceed, and form the probabilities
  auto soften = [&](int c0, int end) {
    if (c0 + 16 * NT > nfree) {
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        const int qi = qw0 + 16 * q + c, seen = visible(qi < p.Nq ? qi : p.Nq - 1), lim = seen < end ? seen : end;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (c0 + 16 * t + 4 * g + r >= lim) s[q][t][r] = -INFINITY;
      }
    }
    bool above = false;
#pragma unroll
    for (int q = 0; q < QT; ++q) above |= top(q) > thr[q];
    if (__builtin_amdgcn_ballot_w64(above) != 0) {
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        const float mnew = fmaxf(mref[q], mul_rounded(xmax(top(q)), scale2));
        const float f = exp2_fast(mref[q] - mnew);
        const bool far = mnew > kNoKey && fabsf(mnew) > kFarRef;
        mref[q] = mnew;
        mul[q] = far ? 1.0f : scale2;
        off[q] = far ? 0.0f : mnew;
        thr[q] = (mnew + (far ? -INFINITY : kGrow)) / scale2;     // (no branch: it would part the loop)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[q][t][r] = far ? mul_rounded(s[q][t][r], scale2) - mnew : s[q][t][r];
        lrun[q] *= f;
#pragma unroll
        for (int vt = 0; vt < NVT; ++vt) o[q][vt] = o[q][vt] * f;
      }
    }
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[q][t][r] = exp2_fast(fmaf(s[q][t][r], mul[q], -off[q]));
          if (CODES && t == 0 && r == 0) sum = s[q][t][r];
          else sum += s[q][t][r];
        }
      lrun[q] += sum;
#pragma unroll
      for (int st = 0; st < NS; ++st) pb[q][st] = pack8(s[q][2 * st], s[q][2 * st + 1]);
    }
  };
  auto phase_end = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
  };

  fetch(p0);
  const Tile k0 = kt, v0 = vt;
  fetch(p0 + 1);
  const Tile k1 = kt, v1 = vt;
  fetch(p0 + 2);
  k0.store(dense_lds + (p0 & (kDenseSlots - 1)) * kDenseSlot<D>, tid);
  v0.store(dense_lds + (p0 & (kDenseSlots - 1)) * kDenseSlot<D> + 64 * LD, tid);
  k1.store(dense_lds + ((p0 + 1) & (kDenseSlots - 1)) * kDenseSlot<D>, tid);
  v1.store(dense_lds + ((p0 + 1) & (kDenseSlots - 1)) * kDenseSlot<D> + 64 * LD, tid);
  __syncthreads();
  matrix(p0 & (kDenseSlots - 1), 0, false);
  if (second) __syncthreads();
  auto step = [&](int i, int end, bool mine) {
    if (mine) soften(first_key(i) + (WK == 2 ? 32 * wk : 0), end);
    // pair i + 2 into the slot of pair i - 2, which both halves left at least a phase ago (the other
    // half may still be reading pairs i - 1 and i)
    commit((i + 2) & (kDenseSlots - 1));
    fetch(i + 3);
    phase_end();
    __builtin_amdgcn_s_setprio(1);
    if (mine) matrix((i + 1) & (kDenseSlots - 1), i & (kDenseSlots - 1), true);
    __builtin_amdgcn_s_setprio(0);
    phase_end();
  };
  for (int i = p0; i < (PART && p1 < nmid ? p1 : nmid); ++i) step(i, mid, true);
  if constexpr (WK == 1) {
    for (int i = PART && p0 > nmid ? p0 : nmid; i < p1; ++i) step(i, nkeys, second);
  }
  if (!second) __syncthreads();

  if constexpr (WK == 2) {
    // the second half's reference, sum and accumulators, merged into the first half's
    f32x4* xo = (f32x4*)dense_lds + (size_t)wq * (QT * (NVT + 1)) * 64 + lane;
    __syncthreads();
    if (wk == 1) {
#pragma unroll
      for (int q = 0; q < QT; ++q) {
#pragma unroll
        for (int vt = 0; vt < NVT; ++vt) xo[(q * (NVT + 1) + vt) * 64] = o[q][vt];
        xo[(q * (NVT + 1) + NVT) * 64] = f32x4{mref[q], lrun[q], 0.f, 0.f};
      }
    }
    __syncthreads();
    if (wk == 1) return;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const f32x4 ml = xo[(q * (NVT + 1) + NVT) * 64];
      const float m = fmaxf(mref[q], ml[0]), f0 = exp2_fast(mref[q] - m), f1 = exp2_fast(ml[0] - m);
      lrun[q] = lrun[q] * f0 + ml[1] * f1;
      mref[q] = m;
#pragma unroll
      for (int vt = 0; vt < NVT; ++vt) o[q][vt] = o[q][vt] * f0 + xo[(q * (NVT + 1) + vt) * 64] * f1;
    }
  }
  if (PART && !own_rows) {
    long long row0 = ((long long)part * parts.heads + bh) * p.Nq;
    if constexpr (PART && CODES)
      if (rest >= 0) row0 = ((long long)part * save.rounds.rest + rest) * WGQ - q0;
    // (hidden for the same reason as below: 12 heads of 4680 queries of 32760 keys in four parts 777 -> 575 us)
    int col = c, row = g;
    if constexpr (CODES && D == 64) asm volatile("" : "+v"(col), "+v"(row));
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      const int qi = qw0 + 16 * q + col;
      const float lsum = xsum(lrun[q]);
      if (qi < p.Nq) {
        float* at = parts.o + (row0 + qi) * D + 4 * row;
#pragma unroll
        for (int vt = 0; vt < NVT; ++vt) *(f32x4*)(at + 16 * vt) = o[q][vt];
        if (row == 0) parts.ml[row0 + qi] = make_float2(mref[q], lsum);
      }
    }
    return;
  }
  u16* Op = (u16*)p.O + b * p.os.batch + hd * p.os.head;
  // (what the stores' addresses are formed from is hidden, or the compiler forms them before the loop and keeps three more
  // registers in memory there: 12 heads of 4680 tokens of 64 features 98 instead of 91 us)
  int col = c;
  if constexpr (SAVE) asm volatile("" : "+v"(col));
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const int qi = qw0 + 16 * q + col;
    const float lsum = xsum(lrun[q]), inv = lsum > 0.f ? 1.0f / lsum : 0.f;
    if (qi < p.Nq) {
      u16* row = Op + (long long)qi * p.os.token + 4 * g;
#pragma unroll
      for (int vt = 0; vt < NVT; ++vt) {
        const f32x4 x = o[q][vt] * inv;
        typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
        *(bf16x4*)(row + 16 * vt) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
      }
      if constexpr (SAVE)
        if (g == 0) save.lse[(long long)bh * p.Nq + qi] = natural_lse(mref[q], lsum);
    }
  }
}

// O from the parts: every part's sum and accumulators against the largest reference.  A thread owns
// four features of a query and has eight parts in flight at once: what it waits for is memory.
template <int D, typename Save>
__global__ __launch_bounds__(256) void k_dense_merge(KParams p, DenseParts parts, int rows, Save save) {
  constexpr int TPR = D / 4, AHEAD = 8;
  const int row = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, f = 4 * (threadIdx.x % TPR);
  if (row >= rows) return;
  float m = kNoKey, lsum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < parts.n; i0 += AHEAD) {
    float2 ml[AHEAD];
    f32x4 po[AHEAD];
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      const size_t at = (size_t)(i0 + e < parts.n ? i0 + e : parts.n - 1) * rows + row;
      ml[e] = parts.ml[at];
      po[e] = *(const f32x4*)(parts.o + at * D + f);
    }
    float top = m;
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) top = fmaxf(top, ml[e].x);
    const float keep = exp2_fast(m - top);
    m = top;
    lsum *= keep;
    o = o * keep;
#pragma unroll
    for (int e = 0; e < AHEAD; ++e)
      if (i0 + e < parts.n) {
        const float w = exp2_fast(ml[e].x - m);
        lsum += ml[e].y * w;
        o = o + po[e] * w;
      }
  }
  const float inv = lsum > 0.f ? 1.0f / lsum : 0.f;
  const f32x4 x = o * inv;
  int bh = row / p.Nq, q = row - bh * p.Nq;
  if constexpr (dense_codes<Save>)
    if (save.rounds.rest > 0) {      // rows of the last round's tiles
      const DenseRounds& r = save.rounds;
      const int nx = (p.Nq + r.queries - 1) / r.queries, at = row / r.queries, unit = r.whole + at;
      bh = unit / nx;
      q = (unit - bh * nx) * r.queries + row - at * r.queries;
      if (q >= p.Nq) return;
    }
  const int b = bh / p.H, hd = bh - b * p.H;
  typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
  *(bf16x4*)((u16*)p.O + b * p.os.batch + hd * p.os.head + (long long)q * p.os.token + f) =
      bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
  if constexpr (dense_codes<Save>) {
    if (f == 0) save.lse[(long long)bh * p.Nq + q] = natural_lse(m, lsum);
  } else if constexpr (!std::is_same<Save, NoSave>::value) {
    if (f == 0) save.lse[row] = natural_lse(m, lsum);
  }
}

template <int D, int QT, int WK, bool PART, typename Save>
hipError_t run_dense(const KParams& kp, int nbh, const DenseParts& parts, const Save& save, hipStream_t s) {
  const auto kernel = k_bf16_dense<D, QT, WK, PART, Save>;
  const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kDenseLds<D>);
  if (e != hipSuccess) return e;
  constexpr int wgq = 16 * QT * kDenseWaves / WK;
  kernel<<<(kp.Nq + wgq - 1) / wgq * nbh * parts.n, kDenseThreads, kDenseLds<D>, s>>>(kp, parts, save);
  if constexpr (PART) {
    const int rows = nbh * kp.Nq, rpw = 256 / (D / 4);
    k_dense_merge<D><<<(rows + rpw - 1) / rpw, 256, 0, s>>>(kp, parts, rows, save);
  }
  return hipGetLastError();
}

inline size_t dense_parts_bytes(int rows, int parts, int d) { return (size_t)rows * parts * (d + 2) * sizeof(float); }

template <int D, bool PART, typename Save>
hipError_t run_dense_d(const KParams& kp, int nbh, int queries, const DenseParts& parts, const Save& save, hipStream_t s) {
  if (queries == 64) return run_dense<D, 1, 2, PART>(kp, nbh, parts, save, s);
  if constexpr (D == 128)
    if (queries == 256) return run_dense<D, 2, 1, PART>(kp, nbh, parts, save, s);
  return run_dense<D, 2, 2, PART>(kp, nbh, parts, save, s);
}
template <typename Save>
hipError_t run_dense_shape(const KParams& kp, int nbh, const DenseShape& shape, const DenseParts& parts, const Save& save, hipStream_t s) {
  if (kp.d == 128)
    return shape.parts > 1 ? run_dense_d<128, true>(kp, nbh, shape.queries, parts, save, s)
                           : run_dense_d<128, false>(kp, nbh, shape.queries, parts, save, s);
  return shape.parts > 1 ? run_dense_d<64, true>(kp, nbh, shape.queries, parts, save, s)
                         : run_dense_d<64, false>(kp, nbh, shape.queries, parts, save, s);
}

}  // namespace

// of a call with `bytes` of scratch (mrt_dense_bf16.hip)
DenseShape dense_call_shape(const KParams& kp, int nbh, size_t bytes, bool save);

}  // namespace mrt
