// Rows into a cache of 8 bits and out of it (mrt_cache8.hpp says what it holds).
//
// Writing: a workgroup, or a wave where a block of tokens is small, owns one block of one (batch, head) of K or V: it
// holds the block's rows in registers, those that are there before the first new one among them, takes their largest
// magnitude, and stores codes.  The scale is the smallest power of two that brings that magnitude to the largest code, found
// from its bits; codes are the nearest, ties to even, of a product with a power of two, which is exact.  Both calls move
// every byte once and are bound by memory: 12 heads of 4680 tokens, e4m3, written in 11.7 us (28.8 MB read, 14.4 written) and read
// in 9.9; 32760 of them in whole numbers read in 52 (101 MB read, 201 written).
#include "mrt_cache8.hpp"

#include <algorithm>

namespace mrt {

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
constexpr int kThreadsCache = 256, kItem = 16;       // codes of an access
// Workgroups along a head's rows: one access a thread up to long runs (4680 rows of 12 heads written, 32760 read, whole numbers,
// by the most: 4096 68 us, 512 74, 256 79, 64 85).
constexpr unsigned kMostReadWgs = 4096;

// 16 numbers of a row, as they come
template <typename T> struct Item;
template <> struct Item<__bf16> {
  u32x4 v[2];
  __device__ inline unsigned bits(int e) const { return e & 1 ? v[e / 8][e / 2 % 4] & 0xffff0000u : v[e / 8][e / 2 % 4] << 16; }
  __device__ inline void set(const bf16x8 (&x)[2]) {
    v[0] = __builtin_bit_cast(u32x4, x[0]);
    v[1] = __builtin_bit_cast(u32x4, x[1]);
  }
};
template <> struct Item<float> {
  u32x4 v[4];
  __device__ inline unsigned bits(int e) const { return v[e / 4][e % 4]; }
  __device__ inline void set(const bf16x8 (&x)[2]) {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e / 4][e % 4] = __builtin_bit_cast(unsigned, (float)x[e / 8][e % 8]);
  }
};
template <typename T> constexpr int kItemAccesses = sizeof(Item<T>) / 16;

constexpr unsigned kInf = 0x7f800000u;

// The exponent byte of a block whose largest magnitude has these bits.
template <bool E4M3>
__device__ inline int exponent_of(unsigned largest) {
  // 448 = 1.75 2^8, 127 = 1.984375 2^6
  const int e = (int)(largest >> 23) - (E4M3 ? 8 : 6) + ((largest & 0x7fffff) > (E4M3 ? 0x600000u : 0x7e0000u));
  return e < kCacheLeast ? kCacheLeast : e > kCacheMost ? kCacheMost : e;
}

// Codes of 16 numbers.  Beyond the largest code (infinities, and numbers beyond 2^127) they are that code; NaN stays one in
// e4m3 and becomes 0 in whole numbers.  (By its bits: the library is compiled without regard to NaN in comparisons.)
template <typename T, bool E4M3>
__device__ inline u32x4 encode(const Item<T>& x, float inverse) {
  u32x4 codes;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    unsigned y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned bits = x.bits(4 * w + e);
      const float z = __builtin_bit_cast(float, bits) * inverse, most = E4M3 ? 448.f : 127.f;
      const float c = fminf(fmaxf(z, -most), most);
      const bool nan = (bits & 0x7fffffffu) > kInf;
      y[e] = nan ? (E4M3 ? 0x7fffffffu : 0u) : __builtin_bit_cast(unsigned, c);
    }
    auto f = [&](int e) { return __builtin_bit_cast(float, y[e]); };
    if constexpr (E4M3) {
      int q = __builtin_amdgcn_cvt_pk_fp8_f32(f(0), f(1), 0, false);
      codes[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f(2), f(3), q, true);
    } else {
      unsigned q = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) q |= ((unsigned)(int)__builtin_rintf(f(e)) & 255u) << (8 * e);
      codes[w] = q;
    }
  }
  return codes;
}

template <bool E4M3>
__device__ inline void decode(u32x4 codes, float scale, bf16x8 (&x)[2]) {
  x[0] = cache8_values<E4M3>(u32x2{codes[0], codes[1]}, scale);
  x[1] = cache8_values<E4M3>(u32x2{codes[2], codes[3]}, scale);
}

// TEAM: threads of a block of tokens.  ITEMS: of a thread.
template <typename T, bool E4M3, int TEAM, int ITEMS>
__global__ __launch_bounds__(kThreadsCache) void k_cache8_write(const Cache8Call c, int touched, int units) {
  constexpr int TEAMS = kThreadsCache / TEAM;
  __shared__ unsigned tops[4];
  const int me = threadIdx.x % TEAM, team = TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0;
  const int unit = blockIdx.x * TEAMS + team;        // (block, head, sequence)
  const Cache8Side& side = c.side[blockIdx.y];
  const int bh = unit / touched, b = bh / c.heads, head = bh - b * c.heads;
  bool runs = unit < units;
  long long at = 0;
  int lo = 0, end = 0, block = 0, first = 0;
  if (runs) {
    at = c.at_each ? c.at_each[b] : c.at;
    const int n = c.tokens_each ? min(max(c.tokens_each[b], 0), c.tokens) : c.tokens;
    lo = (int)min(max(at, 0ll), (long long)c.capacity);
    end = (int)min(max(at + n, 0ll), (long long)c.capacity);
    block = (lo >> c.shift) + unit - bh * touched;
    first = block << c.shift;
    runs = lo < end && first < end;
  }
  if (TEAMS > 1 && !runs) return;                    // (a wave by itself)
  unsigned char* codes = side.codes + b * side.cs.batch + head * side.cs.head;
  unsigned char* exps = side.exps + b * side.exp_batch + head * side.exp_head;
  const T* rows = (const T*)side.rows + b * side.rs.batch + head * side.rs.head;
  const int per = c.d / kItem, items = runs ? per << c.shift : 0;
  const int old = runs && first < lo ? exps[block] : 0;
  // An infinity does not take the scale of a block whose earlier rows are kept: under 2^119 they would be zeros.
  const unsigned largest = first < lo ? kInf - 1 : kInf;
  Item<T> x[ITEMS];
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int item = me + i * TEAM, token = first + item / per, f = kItem * (item % per);
#pragma unroll
    for (int k = 0; k < kItemAccesses<T>; ++k) x[i].v[k] = u32x4{0, 0, 0, 0};
    if (item < items && token < lo) {                // kept
      bf16x8 values[2];
      decode<E4M3>(*(const u32x4*)(codes + (long long)token * side.cs.token + f), cache8_scale(old), values);
      x[i].set(values);
    } else if (item < items && token < end) {
      const u32x4* row = (const u32x4*)(rows + (token - at) * side.rs.token + f);
#pragma unroll
      for (int k = 0; k < kItemAccesses<T>; ++k) x[i].v[k] = row[k];
    }
#pragma unroll
    for (int e = 0; e < kItem; ++e) {
      const unsigned m = x[i].bits(e) & 0x7fffffffu;
      top = max(top, m > largest ? 0u : m);
    }
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) top = max(top, (unsigned)__shfl_xor((int)top, m));
  if constexpr (TEAM > 64) {
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x / 64] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  }
  if (!runs) return;
  const int now = exponent_of<E4M3>(top);
  const float inverse = cache8_scale(254 - now);
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int item = me + i * TEAM, token = first + item / per, f = kItem * (item % per);
    // (kept rows under an unchanged scale have the codes they had)
    if (item < items && token < end && (token >= lo || now != old))
      *(u32x4*)(codes + (long long)token * side.cs.token + f) = encode<T, E4M3>(x[i], inverse);
  }
  if (me == 0) exps[block] = (unsigned char)now;
}

// A thread 16 codes of a row at a time.
template <typename T, bool E4M3>
__global__ __launch_bounds__(kThreadsCache) void k_cache8_read(const Cache8Call c, unsigned items) {
  const Cache8Side& side = c.side[blockIdx.z];
  const int b = blockIdx.y / c.heads, head = blockIdx.y - b * c.heads;
  const unsigned per = (unsigned)c.d / kItem;
  const long long at = c.at_each ? c.at_each[b] : c.at;
  const unsigned char* codes = side.codes + b * side.cs.batch + head * side.cs.head;
  const unsigned char* exps = side.exps + b * side.exp_batch + head * side.exp_head;
  T* rows = (T*)side.rows + b * side.rs.batch + head * side.rs.head;
  for (unsigned item = blockIdx.x * kThreadsCache + threadIdx.x; item < items; item += gridDim.x * kThreadsCache) {
    const unsigned row = item / per, f = kItem * (item - row * per);
    const long long token = at + row;
    u32x4 code = {0, 0, 0, 0};
    unsigned e = 127;
    if (token >= 0 && token < c.capacity) {
      code = *(const u32x4*)(codes + token * side.cs.token + f);
      e = exps[token >> c.shift];
    }
    bf16x8 x[2];
    decode<E4M3>(code, cache8_scale(e), x);
    Item<T> out;
    out.set(x);
    u32x4* to = (u32x4*)(rows + (long long)row * side.rs.token + f);
#pragma unroll
    for (int j = 0; j < kItemAccesses<T>; ++j) to[j] = out.v[j];
  }
}

template <typename T, bool E4M3>
hipError_t write(const Cache8Call& c, hipStream_t s) {
  const int block = 1 << c.shift, items = block * (c.d / kItem);
  // blocks that a run can touch, wherever it begins
  const int touched = c.at_each ? (c.tokens + block - 2) / block + 1 : (c.at + c.tokens - 1) / block - c.at / block + 1;
  const long long units = (long long)touched * c.batch * c.heads;
  if (units > 0x7fffffff) return hipErrorInvalidValue;
  const int per_wg = items <= 256 ? 4 : 1;
  const dim3 grid((unsigned)((units + per_wg - 1) / per_wg), 2);
#define MRT_WRITE(team, n) k_cache8_write<T, E4M3, team, n><<<grid, kThreadsCache, 0, s>>>(c, touched, (int)units)
  if (items <= 64) MRT_WRITE(64, 1);
  else if (items <= 128) MRT_WRITE(64, 2);
  else if (items <= 256) MRT_WRITE(64, 4);
  else if (items <= 512) MRT_WRITE(256, 2);
  else if (items <= 1024) MRT_WRITE(256, 4);
  else MRT_WRITE(256, 8);
#undef MRT_WRITE
  return hipGetLastError();
}

template <typename T, bool E4M3>
hipError_t read(const Cache8Call& c, hipStream_t s) {
  const unsigned items = (unsigned)c.tokens * (c.d / kItem);      // (2^24 x 16 at most)
  const dim3 grid(std::min((items + kThreadsCache - 1) / kThreadsCache, kMostReadWgs), c.batch * c.heads, 2);
  k_cache8_read<T, E4M3><<<grid, kThreadsCache, 0, s>>>(c, items);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache8_write(const Cache8Call& c, bool e4m3, mrt_dtype dtype, hipStream_t s) {
  if (dtype == MRT_F32) return e4m3 ? write<float, true>(c, s) : write<float, false>(c, s);
  return e4m3 ? write<__bf16, true>(c, s) : write<__bf16, false>(c, s);
}
hipError_t launch_cache8_read(const Cache8Call& c, bool e4m3, mrt_dtype dtype, hipStream_t s) {
  if (dtype == MRT_F32) return e4m3 ? read<float, true>(c, s) : read<float, false>(c, s);
  return e4m3 ? read<__bf16, true>(c, s) : read<__bf16, false>(c, s);
}

}  // namespace mrt
