// A cache of keys and values in 8 bits: codes, and a power of two for every block of tokens of a (batch, head).
//
// A power of two, held as its exponent + 127: a code times its scale then is a bf16 number exactly (4 or 7 significant
// bits), which the matrix unit takes as it is, and a scale that has to grow when rows are appended to a block rounds the
// rows that are there by a whole number of halvings: not at all for e4m3 codes that stay normal, and by less than one new
// step in all, however often, for whole numbers (each halving adds half a new step, and halves what was there before).  A scale
// that shrinks again, since the rows behind were replaced, gives nothing back of that.
// Against the scale max / 127 it costs whole numbers up to one bit; e4m3 codes, whose precision is relative, nothing.
#pragma once
#include "mrt_internal.hpp"

namespace mrt {

// Exponents + 127 that are in use: at 3 the smallest code is 2^-133, the smallest bf16 number; at 246 the largest is 1.75 2^127.
constexpr int kCacheLeast = 3, kCacheMost = 246;

namespace {

__device__ inline float cache8_scale(unsigned e) { return __builtin_bit_cast(float, e << 23); }

// 8 codes as bf16 numbers
template <bool E4M3>
__device__ inline __attribute__((ext_vector_type(8))) __bf16 cache8_values(__attribute__((ext_vector_type(2))) unsigned v, float scale) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
  bf16x2 x[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (E4M3) {
      x[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], scale, false);
      x[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], scale, true);
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k)
        x[2 * i + k] = bf16x2{(__bf16)((float)(signed char)(v[i] >> (16 * k)) * scale),
                              (__bf16)((float)(signed char)(v[i] >> (16 * k + 8)) * scale)};
    }
  }
  const bf16x4 lo = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3), hi = __builtin_shufflevector(x[2], x[3], 0, 1, 2, 3);
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

}  // namespace

// What the launchers of mrt_cache8.hip take: one tensor of a cache and the rows it gives or gets.
struct Cache8Side {
  unsigned char* codes;
  unsigned char* exps;
  void* rows;
  mrt_strides cs, rs;               // codes (bytes) and rows (elements)
  long long exp_batch, exp_head;
};
struct Cache8Call {
  Cache8Side side[2];               // keys, values
  int batch, heads, d, capacity, shift;
  int tokens, at;                   // rows of the call, token of the first one ...
  const int *at_each, *tokens_each; // ... or those of every sequence, on the device (null: tokens, at)
};
hipError_t launch_cache8_write(const Cache8Call& c, bool e4m3, mrt_dtype dtype, hipStream_t s);
hipError_t launch_cache8_read(const Cache8Call& c, bool e4m3, mrt_dtype dtype, hipStream_t s);

// The attention over a cache (mrt_dense_cache8.hip).
template <bool E4M3>
hipError_t launch_dense_cache8(const KParams& kp, int nbh, void* workspace, size_t workspace_bytes, const DenseCache8<E4M3>& cache, hipStream_t s);
size_t dense_cache8_workspace_bytes(const KParams& kp, int nbh, int group, bool e4m3);

}  // namespace mrt
