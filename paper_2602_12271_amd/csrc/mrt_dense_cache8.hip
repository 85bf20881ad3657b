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
// their sums at the end; `parts` workgroups share the keys, and a second launch joins theirs.
#include "mrt_dense_bf16.hpp"

#include <algorithm>

namespace mrt {

namespace {

constexpr int kFewWaves = 4, kFewThreads = 64 * kFewWaves, kFewKeys = 32;

// 32 keys and values of a wave, as they come from memory
template <int D>
struct FewTile {
  static constexpr int KP = D / 64;                 // 16-byte pieces of a key that a lane holds
  u32x4 k[2][KP];
  unsigned v[8][D / 64];
  unsigned char ke[2], ve[2];
};

template <int D, bool E4M3, int RT, bool PART>
__global__ __launch_bounds__(kFewThreads, RT == 4 ? 1 : 2) void k_cache8_few(KParams p, DenseParts parts, DenseCache8<E4M3> cache,
                                                                             int row_tiles) {
  constexpr int KP = D / 64, NK = D / 32, NV = D / 16, LD = D + 4;
  extern __shared__ __attribute__((aligned(16))) float few_lds[];      // [wave][row][LD], then [wave][row] references, sums
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  // units that stream the same keys go to one of the eight XCDs
  const int total = gridDim.x, xcd = blockIdx.x & 7;
  const int unit = xcd * (total >> 3) + (xcd < (total & 7) ? xcd : (total & 7)) + (blockIdx.x >> 3);
  const int tile_rows = 16 * RT, rows = cache.group * p.Nq, kv_heads = p.H / cache.group;
  int at = unit;
  const int rt = at % row_tiles;
  at /= row_tiles;
  const int part = PART ? at % parts.n : 0, bk = PART ? at / parts.n : at;
  const int b = bk / kv_heads, kvh = bk - b * kv_heads;
  if (cache.kv_len) p.Nkv = __builtin_amdgcn_readfirstlane(min(max(cache.kv_len[b], 0), p.Nkv));
  const int nkeys = p.Nkv > 0 ? dense_visible(p, p.Nq - 1) : 0, nfree = dense_visible(p, 0);
  const int tiles = (nkeys + kFewKeys - 1) / kFewKeys;
  const int t0 = PART ? (int)((long long)part * tiles / parts.n) : 0, t1 = PART ? (int)((long long)(part + 1) * tiles / parts.n) : tiles;

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
  const auto kr = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)p.K + b * p.ks.batch + kvh * p.ks.head), 0, last * krow + D, 0x00020000);
  const auto vr = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)p.V + b * p.vs.batch + kvh * p.vs.head), 0, last * vrow + D, 0x00020000);
  const int exps = (int)(last >> cache.shift) + 1;
  const auto ker = __builtin_amdgcn_make_buffer_rsrc((void*)(cache.k_exp + b * cache.ke_batch + kvh * cache.ke_head), 0, exps, 0x00020000);
  const auto ver = __builtin_amdgcn_make_buffer_rsrc((void*)(cache.v_exp + b * cache.ve_batch + kvh * cache.ve_head), 0, exps, 0x00020000);
  auto fetch = [&](FewTile<D>& x, int t) {              // (zeros beyond the last key)
    const unsigned key = (unsigned)t * kFewKeys;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x.ke[h] = __builtin_amdgcn_raw_buffer_load_b8(ker, (key + 16 * h + c) >> cache.shift, 0, 0);
      x.ve[h] = __builtin_amdgcn_raw_buffer_load_b8(ver, (key + 16 * h + 4 * g) >> cache.shift, 0, 0);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < KP; ++j) x.k[h][j] = __builtin_amdgcn_raw_buffer_load_b128(kr, (key + 16 * h + c) * krow + 16 * (g + 4 * j), 0, 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned off = (key + 16 * (e / 4) + 4 * g + e % 4) * vrow + D / 16 * c;
      if constexpr (D == 128) {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(vr, off, 0, 0);
        x.v[e][0] = w[0];
        x.v[e][1] = w[1];
      } else {
        x.v[e][0] = __builtin_amdgcn_raw_buffer_load_b32(vr, off, 0, 0);
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
      const float scale = cache8_scale(x.ke[h]);
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const u32x4 w = x.k[h][k / 2];
        const bf16x8 key = cache8_values<E4M3>(k % 2 ? u32x2{w[2], w[3]} : u32x2{w[0], w[1]}, scale);
#pragma unroll
        for (int i = 0; i < RT; ++i) s[i][h] = mfma(key, qv[i][k], k ? s[i][h] : f32x4{0.f, 0.f, 0.f, 0.f});
      }
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
    // values: pairs of features of a key, then pairs of keys of a feature
    const float vs[2] = {cache8_scale(x.ve[0]), cache8_scale(x.ve[1])};
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
    }
  };

  FewTile<D> x, y;
  int t = t0 + wave;
  if (t < t1) fetch(x, t);
  for (; t < t1; t += 2 * kFewWaves) {
    if (t + kFewWaves < t1) fetch(y, t + kFewWaves);
    use(x, t);
    if (t + kFewWaves >= t1) break;
    if (t + 2 * kFewWaves < t1) fetch(x, t + 2 * kFewWaves);
    use(y, t + kFewWaves);
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
      const long long to = (long long)part * parts.heads * p.Nq + out;
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

struct FewShape {
  int rt, row_tiles, parts;      // tiles of 16 rows of a workgroup, workgroups for all rows, for all keys; rt = 0: not this kernel
};

constexpr int kFewQueries = 16;
FewShape few_shape(const KParams& kp, int nbh, int group, bool may_split) {
  FewShape f = {0, 1, 1};
  if (kp.Nq > kFewQueries) return f;
  const int rows = group * kp.Nq;
  f.rt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  f.row_tiles = (rows + 16 * f.rt - 1) / (16 * f.rt);
  const long long wgs = (long long)nbh / group * f.row_tiles, tiles = (dense_visible(kp, kp.Nq - 1) + kFewKeys - 1) / kFewKeys;
  const long long want = (4ll * compute_units() / (f.rt == 4 ? 2 : 1) + wgs - 1) / wgs;
  f.parts = may_split ? (int)std::max(1ll, std::min({want, tiles / 8, 64ll})) : 1;
  return f;
}

template <int D, bool E4M3, int RT>
hipError_t run_few(const KParams& kp, int nbh, const FewShape& f, const DenseParts& parts, const DenseCache8<E4M3>& cache, hipStream_t s) {
  constexpr int lds = kFewWaves * 16 * RT * (D + 4 + 2) * (int)sizeof(float);
  const auto kernel = f.parts > 1 ? k_cache8_few<D, E4M3, RT, true> : k_cache8_few<D, E4M3, RT, false>;
  const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  kernel<<<nbh / cache.group * f.row_tiles * f.parts, kFewThreads, lds, s>>>(kp, parts, cache, f.row_tiles);
  if (f.parts > 1) {
    const int rows = nbh * kp.Nq, rpw = 256 / (D / 4);
    k_dense_merge<D><<<(rows + rpw - 1) / rpw, 256, 0, s>>>(kp, parts, rows, cache);
  }
  return hipGetLastError();
}
template <int D, bool E4M3>
hipError_t run_few_d(const KParams& kp, int nbh, const FewShape& f, const DenseParts& parts, const DenseCache8<E4M3>& cache, hipStream_t s) {
  if (f.rt == 1) return run_few<D, E4M3, 1>(kp, nbh, f, parts, cache, s);
  if (f.rt == 2) return run_few<D, E4M3, 2>(kp, nbh, f, parts, cache, s);
  return run_few<D, E4M3, 4>(kp, nbh, f, parts, cache, s);
}

}  // namespace

size_t dense_cache8_workspace_bytes(const KParams& kp, int nbh, int group) {
  const FewShape f = few_shape(kp, nbh, group, true);
  if (f.rt == 0) return bf16_dense_workspace_bytes(kp, nbh, true);
  return f.parts > 1 ? dense_parts_bytes(kp.Nq * nbh, f.parts, kp.d) : 0;
}

template <bool E4M3>
hipError_t launch_dense_cache8(const KParams& kp, int nbh, void* workspace, size_t workspace_bytes, const DenseCache8<E4M3>& cache, hipStream_t s) {
  const size_t bytes = workspace ? workspace_bytes : 0;
  FewShape f = few_shape(kp, nbh, cache.group, bytes > 0);
  if (f.parts > 1 && bytes < dense_parts_bytes(kp.Nq * nbh, f.parts, kp.d)) f = few_shape(kp, nbh, cache.group, false);
  const DenseShape shape = f.rt ? DenseShape{0, f.parts} : dense_call_shape(kp, nbh, bytes, true);
  const size_t rows = (size_t)kp.Nq * nbh * shape.parts;
  const bool even = dense_visible(kp, 0) == dense_visible(kp, kp.Nq - 1);
  const DenseParts parts = {(float*)workspace, (float2*)((float*)workspace + rows * kp.d), shape.parts, (unsigned)nbh,
                            even ? 0u : (unsigned)nbh * shape.parts};
  if (f.rt) return kp.d == 128 ? run_few_d<128>(kp, nbh, f, parts, cache, s) : run_few_d<64>(kp, nbh, f, parts, cache, s);
  return run_dense_shape(kp, nbh, shape, parts, cache, s);
}
template hipError_t launch_dense_cache8<true>(const KParams&, int, void*, size_t, const DenseCache8<true>&, hipStream_t);
template hipError_t launch_dense_cache8<false>(const KParams&, int, void*, size_t, const DenseCache8<false>&, hipStream_t);

}  // namespace mrt
