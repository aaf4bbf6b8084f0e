// Device helpers of the 8-bit cache (KV8): the conversions between codes and
// floating values, and the matrix products that take them.
//
// Format: e4m3 codes c (OCP: largest 448, no infinity, NaN at 0x7F) and one
// exponent byte E = e + 127 for each (page, KV head, block of BT tokens);
// a stored element is c * 2^e.  e is the least exponent, at least -126, with
// amax <= 448 * 2^e.  A power of two costs no precision next to a free fp32
// scale (the codes are floating point themselves), makes the reconstruction
// c * 2^e exact, and lets a stored code move to another exponent without a
// second rounding except among the subnormal codes.
//
// Codes of a (page, KV head), P * d bytes:
//   K  [P][d]
//   V  [P / 16][d / 64][token / 4 % 4][dim / 4 % 16][dim % 4][token % 4]
// V is a matrix operand as it lies: the value products take, for lane (m, g)
// = (lane % 16, lane / 16), four dims 4 m .. 4 m + 3 of a 64-dim chunk at the
// tokens 4 g .. 4 g + 3 of 16, which are the lane's own 16 bytes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace jfkv {
namespace kv8 {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Four codes to two words of two fp16 (or bf16) values: exact, three mantissa
// bits and at most 2^8.
template <bool BF16>
__device__ __forceinline__ void widen(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  if constexpr (BF16) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, true));
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.0f, true));
  }
}

// Eight codes to one matrix operand.
template <bool BF16>
__device__ __forceinline__ u32x4 widen8(uint32_t a, uint32_t b) {
  uint32_t r0, r1, r2, r3;
  widen<BF16>(a, r0, r1);
  widen<BF16>(b, r2, r3);
  return u32x4{r0, r1, r2, r3};
}

// D = A B + C over 16 x 16 x 32: lane (m, g) feeds row (column) m of A (B) at
// k = 8 g .. 8 g + 7 and receives column m, rows 4 g .. 4 g + 3.
template <bool BF16>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two fp32 values to two halves, nearest even.
template <bool BF16>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
  const f32x2 x = {a, b};
  if constexpr (BF16)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
}

template <bool BF16>
__device__ __forceinline__ float half_to_float(uint32_t bits16) {
  if constexpr (BF16)
    return __uint_as_float(bits16 << 16);
  else
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
}

// The exponent e of a block from its largest magnitude (fp32, finite, >= 0):
// amax = 1.f * 2^x <= 448 * 2^e = 1.75 * 2^(8 + e).
__device__ __forceinline__ int exponent_for(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < -126 ? -126 : e;
}

// 2^e for -126 <= e <= 127; smaller e give 0 (their products round to 0 anyway).
__device__ __forceinline__ float power2(int e) {
  return e < -126 ? 0.0f : __uint_as_float((uint32_t)(e + 127) << 23);
}

// The online softmax over blocks of exponents, in the decode and in the chunk
// attention alike (their files say how it goes).
constexpr float kMargin = 4.0f;  // m is raised where a score exceeds it by more (log2)
constexpr int kRefMax = 10;      // e_v - e_ref stays in 0 .. kRefMax
constexpr int kRefFloor = 80;    // e_ref is not lowered further than this below the largest e_v

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The maximum (sum) over the four lanes that hold a column.
__device__ __forceinline__ float col_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float col_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Accumulators of sum P c count in units of 2^e_ref; their factor where e_ref moves
// from one reference to another.  What has been accumulated never moves down by
// more than 84 (the kernels keep e_ref within that of the largest exponent they have
// met).  Farther down only empty accumulators move, whose first block has a far
// smaller exponent than 0, where e_ref starts (zeros: -126): their factor has to
// stay finite, as zero times infinity is a NaN.
__device__ __forceinline__ float reference_step(int from, int to) {
  const int by = from - to;
  return __builtin_ldexpf(1.0f, by < 100 ? by : 100);
}

// Codes of two scaled values: nearest even, saturated at +-448 (infinities),
// NaN to +0, so that no code is ever a NaN.
__device__ __forceinline__ float code_range(float x) {
  return __builtin_amdgcn_fmed3f(x == x ? x : 0.0f, -448.0f, 448.0f);
}
template <bool HI>
__device__ __forceinline__ uint32_t encode2(float a, float b, uint32_t old) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(code_range(a), code_range(b), (int)old, HI);
}

// Four stored codes times f (a power of two).
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float f) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return encode2<true>(hi.x * f, hi.y * f, encode2<false>(lo.x * f, lo.y * f, 0u));
}

// The larger of two scores (NaN if one is).  As one instruction for up to three
// of them: fmaxf first passes each matrix product's result through another, for
// signalling NaNs.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

}  // namespace kv8
}  // namespace jfkv
