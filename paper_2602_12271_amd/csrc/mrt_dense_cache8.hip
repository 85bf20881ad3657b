// Dense softmax attention over a cache of 8 bits.  Calls of many rows run the kernel of bf16 keys (mrt_dense_bf16.hpp),
// which turns codes into bf16 numbers on their way into LDS; calls of few rows a kernel of their own:
//
//   S^T = K Q^T      P = exp2(scale S - m)      O^T = V^T P^T
//
// for the queries of all heads that share a key head, 16 to a tile of the matrix unit, so that a key is read once.
// A wave takes 32 keys at a time straight from memory into registers, where codes become operands: a lane's keys lie as the
// first product wants them, 16 contiguous features; of the values it loads D / 16 features of the 8 keys whose weights it
// will hold (rows 4g .. 4g + 3 of the two tiles of 16, as the first product leaves them), so that no weight changes lanes, and
// brings pairs of keys of one feature together in registers.  No LDS and no barrier until the four waves of a workgroup join
// their sums at the end; `parts` workgroups share the keys, and a second launch joins theirs.  Memory bounds it: one token of 32
// heads sharing 8, four sequences of 8190 .. 32760 keys, 168 MB, in 34.9 us and 4.1 for the join.
#include "mrt_dense_bf16.hpp"

#include <algorithm>
#include <cmath>

namespace mrt {

namespace {

constexpr int kMostFewParts = 128;
constexpr size_t kMostRoundsBytes = (size_t)192 << 20;
constexpr int kFewWaves = 4, kFewThreads = 64 * kFewWaves, kFewKeys = 32;

// 32 keys and values of a wave, as they come from memory
template <int D>
struct FewTile {
  static constexpr int KP = D / 64;                 // 16-byte pieces of a key that a lane holds
  u32x4 k[2][KP];
  unsigned v[8][D / 64];
  unsigned char ke[2], ve[2];
};

// Which tiles a part of a call with parts has, and where it lies among the parts of all sequences.  Sequences of unequal lengths are
// cut into parts of one length, about the least with which no more than parts.n for every sequence come out, so that the chip is as
// full as with equal ones.  Every workgroup finds it out for itself, from all lengths; whole waves call it.  (us, as many parts for
// every sequence as the longest takes | as its own share: 32 heads sharing 8, lengths 8190 .. 32760, batch of 4, 46.3 | 42.8; one of
// 32760 and seven of 100 60.3 | 21.0; 16 of any up to 16384 73.8 | 61.1; four of 32760, with what the lengths cost, 60.9 | 62.4.)
__device__ inline int few_tiles(KParams p, int len) {
  p.Nkv = min(max(len, 0), p.Nkv);
  return p.Nkv > 0 ? (dense_visible(p, p.Nq - 1) + kFewKeys - 1) / kFewKeys : 0;
}
// op over the lanes up to a lane's own, of numbers that 0 leaves as they are (in 1.2 us less a call than by exchanges through LDS)
template <typename Op>
__device__ inline int lanes_upto(int x, Op op) {
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));      // 1, 2, 4 and 8 lanes down in a row of 16
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));      // the last of a row to every second next one
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));      // the last of two to the next two
  return x;
}
struct FewPart {
  int b;                 // -1: no such part
  int first, n;          // of the sequence's parts, how many
  int tiles;             // of a part
};
// the part `slot`, or with slot = -1 those of sequence b
__device__ inline FewPart few_part(const KParams& p, const DenseParts& parts, const int* kv_len, int tiles, int slot, int b) {
  if (!kv_len) {
    if (slot >= 0) b = slot / parts.n;
    return {b, b * parts.n, parts.n, tiles};
  }
  const int batch = (int)parts.heads / p.H, slots = batch * parts.n, lane = threadIdx.x & 63;
  int sum = 0, most = 0;
  const int len0 = lane < batch ? few_tiles(p, kv_len[lane]) : 0;      // (most batches have no more)
  auto tiles_of = [&](int i) { return i < 64 ? len0 : few_tiles(p, kv_len[i]); };
  for (int i = lane; i < batch; i += 64) {
    const int t = tiles_of(i);
    sum += t;
    most = max(most, t);
  }
  sum = __builtin_amdgcn_readlane(lanes_upto(sum, [](int x, int y) { return x + y; }), 63);
  most = __builtin_amdgcn_readlane(lanes_upto(most, [](int x, int y) { return max(x, y); }), 63);
  const int least = max(kFewWaves, (most + kMostFewParts - 1) / kMostFewParts);
  // (with a part that is not full for every sequence they always fit)
  for (int spare = 0;; spare = spare ? batch : (batch + 1) / 2) {
    const int room = slots - spare;
    tiles = max(least, (sum + room - 1) / room);
    int before = 0;
    FewPart at = {-1, 0, 0, tiles};
    for (int i = lane; i - lane < batch; i += 64) {
      const int n = i < batch ? (tiles_of(i) + tiles - 1) / tiles : 0;
      const int upto = lanes_upto(n, [](int x, int y) { return x + y; }), first = before + upto - n;
      const unsigned long long found = __builtin_amdgcn_ballot_w64(i < batch && (slot >= 0 ? slot >= first && slot < first + n : i == b));
      if (found) {
        const int l = __builtin_ctzll(found);
        at = {i - lane + l, __builtin_amdgcn_readlane(first, l), __builtin_amdgcn_readlane(n, l), tiles};
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (before <= slots || spare == batch) return at;
  }
}

// part_tiles: tiles of 32 keys of a part, where all sequences are as long as the cache.
template <int D, bool E4M3, int RT, bool PART>
__global__ __launch_bounds__(kFewThreads, RT == 4 ? 1 : 2) void k_cache8_few(KParams p, DenseParts parts, DenseCache8<E4M3> cache,
                                                                             int row_tiles, int part_tiles) {
  constexpr int KP = D / 64, NK = D / 32, NV = D / 16, LD = D + 4;
  extern __shared__ __attribute__((aligned(16))) float few_lds[];      // [wave][row][LD], then [wave][row] references, sums
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  // Workgroups reach the eight XCDs in turn: tiles of rows that stream the same keys go to one of them, parts to all.
  const int turn = (int)blockIdx.x >> 3, rt = turn % row_tiles;
  int slot = 8 * (turn / row_tiles) + (int)(blockIdx.x & 7);
  const int tile_rows = 16 * RT, rows = cache.group * p.Nq, kv_heads = p.H / cache.group;
  int b, kvh, part = 0;
  if constexpr (PART) {
    const int slots = (int)parts.heads / p.H * parts.n;
    kvh = slot % kv_heads;
    slot /= kv_heads;
    if (slot >= slots) return;
    const FewPart at = few_part(p, parts, cache.kv_len, part_tiles, slot, 0);
    if (at.b < 0) return;
    b = at.b;
    part = slot - at.first;
    part_tiles = at.tiles;
  } else {
    b = slot / kv_heads;
    kvh = slot - b * kv_heads;
    if (b * p.H >= (int)parts.heads) return;
  }
  if (cache.kv_len) p.Nkv = __builtin_amdgcn_readfirstlane(min(max(cache.kv_len[b], 0), p.Nkv));
  const int nkeys = p.Nkv > 0 ? dense_visible(p, p.Nq - 1) : 0, nfree = dense_visible(p, 0);
  const int tiles = (nkeys + kFewKeys - 1) / kFewKeys;
  const int t0 = PART ? part * part_tiles : 0, t1 = PART ? min(t0 + part_tiles, tiles) : tiles;

  // row r of the tile: query r % Nq of head r / Nq of those that share the keys
  int limit[RT];
  bf16x8 qv[RT][NK];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int r0 = rt * tile_rows + 16 * i + c, r = r0 < rows ? r0 : rows - 1, head = r / p.Nq, q = r - head * p.Nq;
    limit[i] = dense_visible(p, q);
    const u16* Qp = (const u16*)p.Q + b * p.qs.batch + (kvh * cache.group + head) * p.qs.head + q * p.qs.token;
#pragma unroll
    for (int k = 0; k < NK; ++k) qv[i][k] = ld_global_16B(Qp + 16 * (g + 4 * (k / 2)) + 8 * (k % 2));
  }

  const unsigned krow = (unsigned)p.ks.token, vrow = (unsigned)p.vs.token, last = (unsigned)(nkeys - 1);
  const char* Kp = (const char*)p.K + b * p.ks.batch + kvh * p.ks.head;
  const char* Vp = (const char*)p.V + b * p.vs.batch + kvh * p.vs.head;
  const unsigned char* ke = cache.k_exp + b * cache.ke_batch + kvh * cache.ke_head;
  const unsigned char* ve = cache.v_exp + b * cache.ve_batch + kvh * cache.ve_head;
  // a lane's places in a tile; a tile's resource begins at its first key, so that they stay (zeros beyond the last key)
  unsigned koff[2][KP], voff[8];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int j = 0; j < KP; ++j) koff[h][j] = (16 * h + c) * krow + 16 * (g + 4 * j);
#pragma unroll
  for (int e = 0; e < 8; ++e) voff[e] = (16 * (e / 4) + 4 * g + e % 4) * vrow + D / 16 * c;
  auto fetch = [&](FewTile<D>& x, int t) {
    const unsigned key = (unsigned)t * kFewKeys;
    // (what is the same in all lanes has to be known as such, or every load becomes a loop over the resources of the lanes)
    auto from = [&](const char* base, unsigned row) {
      return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (unsigned)__builtin_amdgcn_readfirstlane(key * row)), 0,
                                               __builtin_amdgcn_readfirstlane((last - key) * row + D), 0x00020000);
    };
    const auto kr = from(Kp, krow), vr = from(Vp, vrow);
#pragma unroll
    for (int h = 0; h < 2; ++h) {                       // (a block has 16 tokens at least)
      const unsigned block = __builtin_amdgcn_readfirstlane(min(key + 16 * h, last) >> cache.shift);
      x.ke[h] = ke[block];
      x.ve[h] = ve[block];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < KP; ++j) x.k[h][j] = __builtin_amdgcn_raw_buffer_load_b128(kr, koff[h][j], 0, 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (D == 128) {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(vr, voff[e], 0, 0);
        x.v[e][0] = w[0];
        x.v[e][1] = w[1];
      } else {
        x.v[e][0] = __builtin_amdgcn_raw_buffer_load_b32(vr, voff[e], 0, 0);
      }
    }
  };

  const float scale2 = p.scale * kLog2e;
  f32x4 o[RT][NV];
  float mref[RT], lrun[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    mref[i] = kNoKey;
    lrun[i] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) o[i][v] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto use = [&](const FewTile<D>& x, int t) {
    f32x4 s[RT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float scale = cache8_scale(__builtin_amdgcn_readfirstlane(x.ke[h]));
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const u32x4 w = x.k[h][k / 2];
        const bf16x8 key = cache8_values<E4M3>(k % 2 ? u32x2{w[2], w[3]} : u32x2{w[0], w[1]}, scale);
#pragma unroll
        for (int i = 0; i < RT; ++i) s[i][h] = mfma(key, qv[i][k], k ? s[i][h] : f32x4{0.f, 0.f, 0.f, 0.f});
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    bf16x8 pb[RT];
    const int key = t * kFewKeys;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i][h][r] = mul_rounded(s[i][h][r], scale2);
      if (key + kFewKeys > nfree) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (key + 16 * h + 4 * g + r >= limit[i]) s[i][h][r] = -INFINITY;
      }
      float top = fmaxf(fmaxf(s[i][0][0], s[i][0][1]), fmaxf(s[i][0][2], s[i][0][3]));
      top = fmaxf(top, fmaxf(fmaxf(s[i][1][0], s[i][1][1]), fmaxf(s[i][1][2], s[i][1][3])));
      if (__builtin_amdgcn_ballot_w64(top > mref[i] + kGrow) != 0) {
        const float m = fmaxf(mref[i], xmax(top)), f = exp2_fast(mref[i] - m);
        mref[i] = m;
        lrun[i] *= f;
#pragma unroll
        for (int v = 0; v < NV; ++v) o[i][v] = o[i][v] * f;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[i][h][r] = exp2_fast(s[i][h][r] - mref[i]);
          lrun[i] += s[i][h][r];
        }
      pb[i] = pack8(s[i][0], s[i][1]);
    }
    __builtin_amdgcn_sched_barrier(0);
    // values: pairs of features of a key, then pairs of keys of a feature
    const float vs[2] = {cache8_scale(__builtin_amdgcn_readfirstlane(x.ve[0])), cache8_scale(__builtin_amdgcn_readfirstlane(x.ve[1]))};
#pragma unroll
    for (int w = 0; w < D / 64; ++w) {
      unsigned pair[2][8];                              // features 4w, 4w + 1 and 4w + 2, 4w + 3 of each key
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bf16x8 y = cache8_values<E4M3>(u32x2{x.v[e][w], 0}, vs[e / 4]);
        const u32x4 bits = __builtin_bit_cast(u32x4, y);
        pair[0][e] = bits[0];
        pair[1][e] = bits[1];
      }
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        u32x4 a;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          a[e] = __builtin_amdgcn_perm(pair[f / 2][2 * e + 1], pair[f / 2][2 * e], f % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int i = 0; i < RT; ++i) o[i][4 * w + f] = mfma(__builtin_bit_cast(bf16x8, a), pb[i], o[i][4 * w + f]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // two tiles by turns: one is loaded while the other is used (three or four, at the price of registers, measured no faster)
  FewTile<D> x[2];
  int t = t0 + wave;
  if (t < t1) fetch(x[0], t);
  for (; t < t1; t += 2 * kFewWaves) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = t + i * kFewWaves, next = at + kFewWaves;
      if (next < t1) fetch(x[1 - i], next);
      if (at < t1) use(x[i], at);
    }
  }

  // the waves' sums, against the largest reference
  float* mine = few_lds + (size_t)wave * tile_rows * LD;
  float* ml = few_lds + (size_t)kFewWaves * tile_rows * LD;            // [wave][row][2]
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const float sum = xsum(lrun[i]);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int v = 0; v < NV; v += 4)
        *(f32x4*)(mine + (16 * i + c) * LD + NV * (4 * g + r) + v) = f32x4{o[i][v][r], o[i][v + 1][r], o[i][v + 2][r], o[i][v + 3][r]};
    if (g == 0) *(float2*)(ml + 2 * (wave * tile_rows + 16 * i + c)) = make_float2(mref[i], sum);
  }
  __syncthreads();
  for (int j = tid; j < tile_rows * (D / 4); j += kFewThreads) {
    const int row = j / (D / 4), f = 4 * (j - row * (D / 4)), r = rt * tile_rows + row;
    if (r >= rows) break;
    float2 w[kFewWaves];
    float m = kNoKey, sum = 0.f;
#pragma unroll
    for (int k = 0; k < kFewWaves; ++k) {
      w[k] = *(const float2*)(ml + 2 * (k * tile_rows + row));
      m = fmaxf(m, w[k].x);
    }
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kFewWaves; ++k) {
      const float by = exp2_fast(w[k].x - m);
      sum += w[k].y * by;
      acc = acc + *(const f32x4*)(few_lds + (size_t)(k * tile_rows + row) * LD + f) * by;
    }
    const int head = r / p.Nq, q = r - head * p.Nq, hd = kvh * cache.group + head;
    const long long out = ((long long)b * p.H + hd) * p.Nq + q;
    if constexpr (PART) {
      const long long to = ((long long)slot * p.H + hd) * p.Nq + q;
      *(f32x4*)(parts.o + to * D + f) = acc;
      if (f == 0) parts.ml[to] = make_float2(m, sum);
    } else {
      const f32x4 z = acc * (sum > 0.f ? 1.0f / sum : 0.f);
      typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
      *(bf16x4*)((u16*)p.O + b * p.os.batch + hd * p.os.head + (long long)q * p.os.token + f) =
          bf16x4{(__bf16)z[0], (__bf16)z[1], (__bf16)z[2], (__bf16)z[3]};
      if (f == 0) cache.lse[out] = natural_lse(m, sum);
    }
  }
}

// O from the parts of few rows: a workgroup a row, whose threads take four features of every eighth (or sixteenth) part, all
// of them under way at once.
template <int D, bool E4M3>
__global__ __launch_bounds__(256) void k_cache8_join(KParams p, DenseParts parts, DenseCache8<E4M3> cache, int part_tiles) {
  constexpr int TPR = D / 4, RUNS = 256 / TPR, MOST = kMostFewParts / RUNS;
  __shared__ __attribute__((aligned(16))) float sums[RUNS][D + 4];
  __shared__ float2 mls[RUNS];
  const int row = blockIdx.x, bh = row / p.Nq, q = row - bh * p.Nq, b = bh / p.H, hd = bh - b * p.H;
  const FewPart at = few_part(p, parts, cache.kv_len, part_tiles, -1, b);
  const int n = at.n;
  const int run = threadIdx.x / TPR, f = 4 * (threadIdx.x % TPR);
  const size_t rows = (size_t)p.H * p.Nq, row0 = at.first * rows + (size_t)hd * p.Nq + q;
  float2 ml[MOST];
  f32x4 po[MOST];
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const int part = run + RUNS * i;
    ml[i] = make_float2(kNoKey, 0.f);
    po[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (part < n) {
      ml[i] = parts.ml[row0 + part * rows];
      po[i] = *(const f32x4*)(parts.o + (row0 + part * rows) * D + f);
    }
  }
  float m = kNoKey, sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < MOST; ++i) m = fmaxf(m, ml[i].x);
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const float w = exp2_fast(ml[i].x - m);
    sum += ml[i].y * w;
    o = o + po[i] * w;
  }
  *(f32x4*)&sums[run][f] = o;
  if (f == 0) mls[run] = make_float2(m, sum);
  __syncthreads();
  if (threadIdx.x >= TPR) return;
  m = kNoKey;
  sum = 0.f;
  o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < RUNS; ++i) m = fmaxf(m, mls[i].x);
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    const float w = exp2_fast(mls[i].x - m);
    sum += mls[i].y * w;
    o = o + *(const f32x4*)&sums[i][f] * w;
  }
  const f32x4 x = o * (sum > 0.f ? 1.0f / sum : 0.f);
  typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
  *(bf16x4*)((u16*)p.O + b * p.os.batch + hd * p.os.head + (long long)q * p.os.token + f) =
      bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
  if (f == 0) cache.lse[row] = natural_lse(m, sum);
}

struct FewShape {
  int rt, row_tiles, parts;      // tiles of 16 rows of a workgroup, workgroups for all rows, for all keys; rt = 0: not this kernel
  int part_tiles;
};

FewShape few_shape(const KParams& kp, int nbh, int group, bool may_split, bool lengths) {
  FewShape f = {0, 1, 1, 0};
  if (kp.Nq > 32) return f;
  const int rows = group * kp.Nq;
  f.rt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  f.row_tiles = (rows + 16 * f.rt - 1) / (16 * f.rt);
  const long long wgs = (long long)nbh / group * f.row_tiles;
  // The kernel of many rows takes 64 queries of a head at a time, whose keys it has in LDS once (us, that one | this one: 12
  // heads over 4680 keys, 12 queries 17.5 | 12.9, 32 18.1 | 16.5, 48 19.0 | 18.8; 32 sharing 8 over 8192 keys 28.4 | 19.1, 29.8 | 25.8, 30.9 |
  // 30.4; over 2048 keys, batch of 8, where tiles fill the chip without sharing keys, 36.8 | 25.5, 24 queries 36.7 | 38.7, 32 38.1 | 43.8).
  if (kp.Nq > 16 && wgs > 64) return {0, 1, 1, 0};
  const long long tiles = (dense_visible(kp, kp.Nq - 1) + kFewKeys - 1) / kFewKeys;
  // As many workgroups as the chip holds at once (two a compute unit, one of 64 rows), each with a tile for every wave.  us by the
  // number of parts: 12 heads 10 34.6, 20 25.5, 42 25.2, 64 26.6; 8 key heads, 4096 keys, 8 10.3, 16 9.2, 32 8.3, 64 9.5; one of 32760 keys 32
  // 13.5, 64 11.1, 96 10.3; 32 heads of 2048 keys, batch of 64, 1 199, 2 210, 8 226; 300 keys 1 6.3, 2 8.2, 6 7.2.
  // Few keys are not parted: the second launch costs 5 us of host time besides (us, parted | not: 8 heads sharing 2, batch of 2, 500 keys
  // 7.6 | 7.3, 1000 7.6 | 10.0; 16 heads of 64 features 700 7.5 | 6.3, 1000 7.2 | 7.1, 1400 7.3 | 8.5).
  const long long batch = nbh / kp.H;
  long long want = 2ll * compute_units() / (f.rt == 4 ? 2 : 1) / wgs;
  // Sequences of lengths of their own are cut where whole ones fill the chip, too: the longest would keep a part of it busy for long
  // (us, whole | three parts a sequence, 32 heads sharing 8, batch of 64, lengths 8192 and 63 of 300 60 | 30, any up to 8192 137 | 121,
  // any of 4096 .. 8192 160 | 167, all 8192 195 | 210; of 128, where whole ones take turns, up to 4096 123 | 134).
  if (lengths && want == 1 && batch > 1 && batch <= 256) want = 3;
  const long long n = may_split && tiles > (kp.d == 64 ? 32 : 16) && tiles * batch < 1ll << 30 ? std::max(1ll, std::min({want, tiles / kFewWaves, (long long)kMostFewParts})) : 1;
  f.part_tiles = (int)((tiles + n - 1) / n);
  f.parts = (int)((tiles + f.part_tiles - 1) / f.part_tiles);
  return f;
}

template <int D, bool E4M3, int RT>
hipError_t run_few(const KParams& kp, int nbh, const FewShape& f, const DenseParts& parts, const DenseCache8<E4M3>& cache, hipStream_t s) {
  constexpr int lds = kFewWaves * 16 * RT * (D + 4 + 2) * (int)sizeof(float);
  const auto kernel = f.parts > 1 ? k_cache8_few<D, E4M3, RT, true> : k_cache8_few<D, E4M3, RT, false>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<(nbh / cache.group * f.parts + 7) / 8 * 8 * f.row_tiles, kFewThreads, lds, s>>>(kp, parts, cache, f.row_tiles, f.part_tiles);
  if (f.parts > 1) k_cache8_join<D><<<nbh * kp.Nq, 256, 0, s>>>(kp, parts, cache, f.part_tiles);
  return hipGetLastError();
}
template <int D, bool E4M3>
hipError_t run_few_d(const KParams& kp, int nbh, const FewShape& f, const DenseParts& parts, const DenseCache8<E4M3>& cache, hipStream_t s) {
  if (f.rt == 1) return run_few<D, E4M3, 1>(kp, nbh, f, parts, cache, s);
  if (f.rt == 2) return run_few<D, E4M3, 2>(kp, nbh, f, parts, cache, s);
  return run_few<D, E4M3, 4>(kp, nbh, f, parts, cache, s);
}

// The shape of a call of many rows that all see the same keys: queries of a workgroup, and workgroups that share the keys of
// every tile of queries, or of those of the last round only (DenseRounds), where tiles beside full rounds would leave a part of
// the chip idle.  A model of microseconds: rounds of as many workgroups as the chip holds (128 features: one a compute unit; 64:
// two, with a lower cost where there is one), each of its steps of 64 keys and a beginning and an end; the launch that joins
// parts, and their bytes, written and read.  Fitted to 40 shapes of 1 to 40 heads and 576 to 32760 keys, each timed with up to 35
// ways; us | model: 12 heads of 1560 queries of 32760 keys, 256 queries shared by three 330 | 321, one by one 831 | 879; 16 heads of
// 4680 of 14040, 256 whole rounds and 48 tiles shared by five 494 | 491, by four 505 | 507, all shared by three 568, one by one
// 755 | 766.  (Two workgroups of unequal length for every tile of one incomplete round, so that units without a tile take the shorter
// ones by turns, measured 894 us where one by one takes 856: 228 tiles of 512 steps.)
// Where sequences have lengths of their own the host does not know them: 128 features, a third of what equal ones would take and two
// thirds of what is left if half the work is missing and the rest in pieces of the longest one (us, as equal ones | so: 12 heads of
// 1560 queries, batch of 4, keys 32760, 20000, 9000, 3000 904 | 640 .. 680, all 32760 1276 | 1337; 8 heads of 780 queries of 9360 and 300
// keys 82 | 72; 4 heads of 576 of 4680, 100, 1000, 200 50 | 45.  64 features gained nothing).
struct RoundsShape {
  DenseRounds r;         // rest = 0: no tiles of their own kind
  int parts;             // 0: no call of this kind
  size_t bytes;
};
RoundsShape rounds_shape(const KParams& kp, int nbh, bool e4m3, size_t most_bytes, bool lengths) {
  RoundsShape best = {{0, 0, 0}, 0, 0};
  if (dense_visible(kp, 0) != dense_visible(kp, kp.Nq - 1)) return best;
  const bool wide = kp.d == 128;
  const long long steps = (dense_visible(kp, 0) + 63) / 64, slots = compute_units() * (wide ? 1ll : 2ll);
  double least = 0;
  for (int i = 0, queries = 64; queries <= (wide ? 256 : 128); queries *= 2, ++i) {
    static const double full_step[2][2][3] = {{{0.90, 1.14, 1.69}, {1.13, 1.43, 1.92}}, {{0.66, 1.17}, {0.99, 1.38}}};
    static const double lone_step[2][2] = {{0.54, 0.78}, {0.62, 0.92}};
    const long long units = (long long)((kp.Nq + queries - 1) / queries) * nbh;
    if (units > 0xffffff) continue;
    auto time = [&](long long wgs, long long n, bool split) {       // `wgs` workgroups of n steps
      const long long whole = wgs / slots, rest = wgs % slots;
      const double full = full_step[!wide][!e4m3][i] * (wide || split || queries == 64 ? 1.0 : 1.06), lone = wide ? full : lone_step[!e4m3][i];
      const double edge = wide ? 9.0 : 3.0;             // (two beside each other hide each other's)
      return whole * (n * full + edge) + (rest ? n * (2 * rest > slots ? full : lone) + edge : 0.0);
    };
    auto look = [&](long long rest, int parts) {        // the tiles that `parts` workgroups share, of `units`
      const size_t bytes = parts > 1 ? dense_parts_bytes(rest == units ? kp.Nq * nbh : (int)rest * queries, parts, kp.d) : 0;
      if (bytes > most_bytes || bytes > kMostRoundsBytes) return;
      double us = time(units - rest, steps, parts > 1) + time(rest * parts, (steps + parts - 1) / parts, parts > 1);
      if (lengths && wide && rest == units) {
        const double piece = time(1, (steps + parts - 1) / parts, parts > 1);
        us = (us + 2 * std::max(piece, 0.5 * piece * units * parts / slots)) / 3;
      }
      if (parts > 1) us = 1.03 * (us + (wide ? 5.5 : 4.0) + 2 * bytes / 5.0e6);       // (it has to promise something)
      if (least > 0 && us >= least) return;
      least = us;
      best = {{(int)(units - rest), (int)rest, queries}, parts, bytes};
    };
    look(units, 1);
    for (int parts = 2; parts <= 32 && 4 * parts <= steps && units * parts <= 6 * slots; ++parts) look(units, parts);
    if (const long long rest = units % slots; rest > 0 && rest < units)
      for (int parts = 2; parts <= kMostFewParts && 4 * parts <= steps && rest * parts <= slots; ++parts) look(rest, parts);
  }
  if (best.r.whole == 0) best.r.rest = 0;               // all tiles alike: the launches of every dense call
  return best;
}

template <int D, bool E4M3, int QT, int WK>
hipError_t run_rounds(const KParams& kp, int nbh, const RoundsShape& shape, const DenseParts& parts, DenseCache8<E4M3> cache, hipStream_t s) {
  const auto kernel = k_bf16_dense<D, QT, WK, true, DenseCache8<E4M3>>;
  const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kDenseLds<D>);
  if (e != hipSuccess) return e;
  cache.rounds = shape.r;
  kernel<<<shape.r.whole + shape.r.rest * shape.parts, kDenseThreads, kDenseLds<D>, s>>>(kp, parts, cache);
  const int rows = shape.r.rest * shape.r.queries, rpw = 256 / (D / 4);
  k_dense_merge<D><<<(rows + rpw - 1) / rpw, 256, 0, s>>>(kp, parts, rows, cache);
  return hipGetLastError();
}
template <bool E4M3>
hipError_t run_rounds(const KParams& kp, int nbh, const RoundsShape& shape, const DenseParts& parts, const DenseCache8<E4M3>& cache, hipStream_t s) {
  if (kp.d == 64)
    return shape.r.queries == 64 ? run_rounds<64, E4M3, 1, 2>(kp, nbh, shape, parts, cache, s) : run_rounds<64, E4M3, 2, 2>(kp, nbh, shape, parts, cache, s);
  if (shape.r.queries == 64) return run_rounds<128, E4M3, 1, 2>(kp, nbh, shape, parts, cache, s);
  return shape.r.queries == 128 ? run_rounds<128, E4M3, 2, 2>(kp, nbh, shape, parts, cache, s) : run_rounds<128, E4M3, 2, 1>(kp, nbh, shape, parts, cache, s);
}

// What a call with `bytes` of scratch does.
struct Cache8Shape {
  FewShape few;
  RoundsShape rounds;    // rest = 0: the dense shape's
  DenseShape dense;
  size_t bytes;          // of parts
};
Cache8Shape cache8_shape(const KParams& kp, int nbh, int group, bool e4m3, size_t bytes, bool lengths) {
  Cache8Shape c;
  c.few = few_shape(kp, nbh, group, bytes > 0, lengths);
  c.rounds = {{0, 0, 0}, 0, 0};
  c.dense = {0, 1};
  c.bytes = 0;
  if (c.few.rt) {
    c.bytes = c.few.parts > 1 ? dense_parts_bytes(kp.Nq * nbh, c.few.parts, kp.d) : 0;
    return c.bytes > bytes ? cache8_shape(kp, nbh, group, e4m3, 0, lengths) : c;
  }
  c.rounds = rounds_shape(kp, nbh, e4m3, bytes, lengths && nbh > kp.H && nbh / kp.H <= 64);
  c.dense = c.rounds.parts ? DenseShape{c.rounds.r.queries, c.rounds.parts} : dense_call_shape(kp, nbh, bytes, true);
  c.bytes = c.rounds.r.rest ? c.rounds.bytes : c.dense.parts > 1 ? dense_parts_bytes(kp.Nq * nbh, c.dense.parts, kp.d) : 0;
  return c;
}

}  // namespace

size_t dense_cache8_workspace_bytes(const KParams& kp, int nbh, int group, bool e4m3) {
  return std::max(cache8_shape(kp, nbh, group, e4m3, ~(size_t)0, false).bytes, cache8_shape(kp, nbh, group, e4m3, ~(size_t)0, true).bytes);
}

template <bool E4M3>
hipError_t launch_dense_cache8(const KParams& kp, int nbh, void* workspace, size_t workspace_bytes, const DenseCache8<E4M3>& cache, hipStream_t s) {
  const Cache8Shape c = cache8_shape(kp, nbh, cache.group, E4M3, workspace ? workspace_bytes : 0, cache.kv_len != nullptr);
  const int n = c.few.rt ? c.few.parts : c.dense.parts;
  const size_t rows = (c.rounds.r.rest ? (size_t)c.rounds.r.rest * c.rounds.r.queries : (size_t)kp.Nq * nbh) * n;
  const bool even = dense_visible(kp, 0) == dense_visible(kp, kp.Nq - 1);
  const DenseParts parts = {(float*)workspace, (float2*)((float*)workspace + rows * kp.d), n, (unsigned)nbh, even ? 0u : (unsigned)nbh * n};
  if (c.few.rt) return kp.d == 128 ? run_few_d<128>(kp, nbh, c.few, parts, cache, s) : run_few_d<64>(kp, nbh, c.few, parts, cache, s);
  if (c.rounds.r.rest) return run_rounds(kp, nbh, c.rounds, parts, cache, s);
  DenseCache8<E4M3> ordered = cache;
  const int batch = nbh / kp.H;
  if (cache.kv_len && batch > 1 && batch <= 64 && even) ordered.by_length = batch;
  return run_dense_shape(kp, nbh, c.dense, parts, ordered, s);
}
template hipError_t launch_dense_cache8<true>(const KParams&, int, void*, size_t, const DenseCache8<true>&, hipStream_t);
template hipError_t launch_dense_cache8<false>(const KParams&, int, void*, size_t, const DenseCache8<false>&, hipStream_t);

}  // namespace mrt
