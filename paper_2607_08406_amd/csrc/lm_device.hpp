// What the operators over requests read of a request, and values of 8, 16 and 32 bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.hpp"
#include "mca_lm.h"

namespace mca {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Cached tokens of request r that count.
__device__ __forceinline__ int cached_of(const mca_tree_attention_args& a, int r) {
  const int most = (int)min((int64_t)a.max_len, (int64_t)a.max_blocks * a.block_size);
  return max(0, min(a.lengths[r], most));
}
// Request r's rows; false if there are none or they are out of range.
__device__ __forceinline__ bool rows_of(const mca_tree_attention_args& a, int r, int* first, int* n) {
  const int64_t f = a.offsets[r], e = a.offsets[r + 1];
  *first = (int)f;
  *n = (int)(e - f);
  return f >= 0 && e > f && e <= a.n_rows && e - f <= a.max_nodes;
}

// Values of 8 bits (e4m3): the low or high two of a word, or all four, times a power of
// two, exactly unless they pass the type's range.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(min(max(byte, 1u), 254u) << 23); }
template <int TYPE, bool HIGH>
__device__ __forceinline__ uint32_t wide2(uint32_t codes, float scale) {
  if constexpr (TYPE == MCA_TYPE_BF16)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HIGH));
}
template <bool HIGH>
__device__ __forceinline__ u32x2 wide2_f32(uint32_t codes, float scale) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, HIGH));
}
// 16 bytes of TYPE from 16 / EL codes
template <int TYPE>
__device__ __forceinline__ u32x4 wide_part(const uint32_t* codes, float scale) {
  if constexpr (TYPE == MCA_TYPE_F32) {
    const u32x2 a = wide2_f32<false>(codes[0], scale), b = wide2_f32<true>(codes[0], scale);
    return u32x4{a[0], a[1], b[0], b[1]};
  } else {
    return u32x4{wide2<TYPE, false>(codes[0], scale), wide2<TYPE, true>(codes[0], scale), wide2<TYPE, false>(codes[1], scale),
                 wide2<TYPE, true>(codes[1], scale)};
  }
}
template <int BYTES>
__device__ __forceinline__ void load_codes(const char* p, uint32_t* out) {
  if constexpr (BYTES == 2) {
    out[0] = gload((const uint16_t*)p);
  } else if constexpr (BYTES == 4) {
    out[0] = gload((const uint32_t*)p);
  } else if constexpr (BYTES == 8) {
    const u32x2 v = gload((const u32x2*)p);
    out[0] = v[0];
    out[1] = v[1];
  } else {
    const u32x4 v = gload((const u32x4*)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = v[i];
  }
}

// Values of a type.
template <int TYPE>
struct Elem {
  static constexpr int kSize = 2, kPer = 8;  // bytes, values of 16 bytes
  typedef uint16_t Raw;
};
template <>
struct Elem<MCA_TYPE_F32> {
  static constexpr int kSize = 4, kPer = 4;
  typedef uint32_t Raw;
};
template <int TYPE>
__device__ __forceinline__ float to_f32(typename Elem<TYPE>::Raw x) {
  if constexpr (TYPE == MCA_TYPE_F32) return __uint_as_float(x);
  if constexpr (TYPE == MCA_TYPE_BF16) return __uint_as_float((uint32_t)x << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)x);
}
template <int TYPE>
__device__ __forceinline__ typename Elem<TYPE>::Raw from_f32(float x) {
  if constexpr (TYPE == MCA_TYPE_F32) return __float_as_uint(x);
  if constexpr (TYPE == MCA_TYPE_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
  return __builtin_bit_cast(uint16_t, (_Float16)x);
}
template <int TYPE>
__device__ __forceinline__ void unpack(u32x4 x, float (&f)[Elem<TYPE>::kPer]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TYPE == MCA_TYPE_F32) {
      f[i] = __uint_as_float(x[i]);
    } else {
      f[2 * i] = to_f32<TYPE>((uint16_t)(x[i] & 0xffff));
      f[2 * i + 1] = to_f32<TYPE>((uint16_t)(x[i] >> 16));
    }
  }
}

// Exponentials and logarithms of 64 bits (the library's are made for all numbers).
// exp(x) of N numbers of at most 700, to 2^-47: 2^n times the series of exp in the rest,
// which is at most ln 2 / 2, to its 11th power.  For x below -707 it is 0
// (results below 2^-1020), NaN stays.
// n comes from the last bits of x / ln 2 + 1.5 2^52 and goes into the exponent as bits:
// conversions, roundings and ldexp of 64 bits take four times as long as a sum.  The steps
// of several go side by side: one by one, each would wait for the one before.
template <int N>
__device__ __forceinline__ void exps_of(double (&x)[N]) {
  constexpr double kInvLn2 = 1.4426950408889634074, kLn2 = 0.69314718055994530942, kLn2Rest = 2.3190468138462996e-17;
  constexpr double kBits = 0x1.8p52;
  constexpr double kOver[12] = {1.0,          1.0,           1.0 / 2,        1.0 / 6,         1.0 / 24,         1.0 / 120,
                                1.0 / 720,    1.0 / 5040,    1.0 / 40320,    1.0 / 362880,    1.0 / 3628800,    1.0 / 39916800};  // 1 / k!
  double t[N], r[N], y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = fma(x[i], kInvLn2, kBits);
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = fma(t[i] - kBits, -kLn2, x[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = fma(t[i] - kBits, -kLn2Rest, r[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = kOver[11];
#pragma unroll
  for (int k = 10; k >= 0; --k) {
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = fma(y[i], r[i], kOver[k]);
    if constexpr (N > 1) __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t n = (uint32_t)__builtin_bit_cast(uint64_t, t[i]);
    const uint64_t bits = __builtin_bit_cast(uint64_t, y[i]) + ((uint64_t)(n << 20) << 32);
    x[i] = x[i] < -707.0 ? 0.0 : __builtin_bit_cast(double, bits);
  }
}
__device__ __forceinline__ double exp_of(double x) {
  double y[1] = {x};
  exps_of(y);
  return y[0];
}
// log(x) of a number that is normal in 32 bits, to 2^-45: its 32-bit logarithm l and the
// logarithm of x exp(-l), which is next to 1.
__device__ __forceinline__ double log_of(double x) {
  const double l = 0.69314718055994530942 * (double)__builtin_amdgcn_logf((float)x);
  const double y = fma(x, exp_of(-l), -1.0);
  return l + y * fma(y, -0.5, 1.0);
}

}  // namespace mca
