// Microscaled 4-bit floating point on gfx950: operand types, register layouts and conversions shared by the mx4_ kernels.
#pragma once
#include "dla_common.hpp"
#include "../../include/dla.h"

namespace dla {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4u_t __attribute__((ext_vector_type(4), aligned(4)));  // 16 bytes from any dword

constexpr int kMxStep = 128;                     // terms of the sum per scaled MFMA step; rows are padded to it
constexpr int64_t kMxMaxLd = (int64_t)1 << 22;   // bytes of a row: offsets inside a tile are 32-bit

struct Mx4View {
  const uint8_t* q;
  const uint8_t* s;
  int64_t ldq, lds;
  int rows;
};

template <dla_dtype DT>
struct MxType;
template <>
struct MxType<DLA_F32> {
  using type = float;
  static constexpr int kTerms = 3;  // 24 bits of mantissa as bf16 terms of 8
};
template <>
struct MxType<DLA_BF16> {
  using type = __bf16;
  static constexpr int kTerms = 1;
};
template <>
struct MxType<DLA_F16> {
  using type = _Float16;
  static constexpr int kTerms = 2;  // 11 bits
};

// 16 x 16 += (16 x 128) * (128 x 16).  Lane l holds 32 neighbouring terms of row l % 16 of A (of column l % 16 of B), those of
// block l / 16, low nibble first, and the block's scale in the low byte of sa (sb); register v of lane l of the result is
// row 4 (l / 16) + v, column l % 16.  Checked against the hardware with all codes and scales, as is that scale 255
// gives NaN and scale 0 is 2^-127.
__device__ __forceinline__ float4_t mx_mma16(i32x4_t a, i32x4_t b, float4_t c, int sa, int sb) {
  const i32x8_t a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 0, sa, 0, sb);
}

// 32 x 32 += (32 x 64) * (64 x 32): lane l holds 32 terms of row l % 32 of A (column l % 32 of B), those of block l / 32; register v of
// lane l of the result is row 8 (v / 4) + 4 (l / 32) + v % 4, column l % 32.  The scales are byte OP (0 .. 3) of sa and sb.
template <int OP>
__device__ __forceinline__ f32x16_t mx_mma32(i32x4_t a, i32x4_t b, f32x16_t c, int sa, int sb) {
  const i32x8_t a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b8, c, 4, 4, OP, sa, OP, sb);
}

// Eight elements (one dword, low nibble first) times the scale, which is exact in bf16 up to the type's range.
__device__ __forceinline__ bf16x8_t mx_values(unsigned int w, float scale) {
  union {
    bf16x2_t p[4];
    bf16x8_t v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return u.v;
}

// Eight elements without their scale.
__device__ __forceinline__ f16x8_t mx_values_f16(unsigned int w) {
  union {
    f16x2_t p[4];
    f16x8_t v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3);
  return u.v;
}

// a's upper 32 lanes for b's lower 32; a's odd rows of 16 lanes for b's even ones.  Both on the pairs of four registers turn register
// and row over.
__device__ __forceinline__ void swap_halves(unsigned int& a, unsigned int& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
__device__ __forceinline__ void swap_rows(unsigned int& a, unsigned int& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// The value x, or what is there plus x, rounded once to element `at` of a matrix of type dt.
template <typename T>
__device__ __forceinline__ void store_value_as(void* c, int64_t at, float x, bool onto) {
  T* const p = static_cast<T*>(c) + at;
  *p = (T)(onto ? (float)*p + x : x);
}
__device__ __forceinline__ void store_value(void* c, int64_t at, float x, dla_dtype dt, bool onto) {
  if (dt == DLA_F32)
    store_value_as<float>(c, at, x, onto);
  else if (dt == DLA_BF16)
    store_value_as<__bf16>(c, at, x, onto);
  else
    store_value_as<_Float16>(c, at, x, onto);
}

// The scale in the low byte of s as the conversions take it: the float whose exponent field it is.  255 stands for a NaN there too,
// and 0 for 2^-127.
__device__ __forceinline__ float mx_scale(unsigned int s) { return __uint_as_float(s << 23 & 0x7f800000u); }

// Its value: 1 with that scale.
__device__ __forceinline__ float mx_scale_value(unsigned int s) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(0x22u, mx_scale(s), 0)[0]; }

// The bf16 terms of x, which add up to it exactly: each takes the leading 8 bits of what the ones before it left (truncated, so
// that the first cannot overflow).  What is not finite is the first term alone; a NaN stays one.
template <int TERMS>
__device__ __forceinline__ void mx_terms(float x, unsigned short* t) {
  unsigned int bits = __float_as_uint(x);
  const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
  if (!finite && (bits & 0x007fffffu)) bits |= 0x00400000u;
  t[0] = (unsigned short)(bits >> 16);
  float rest = finite ? x - __uint_as_float(bits & 0xffff0000u) : 0.0f;
#pragma unroll
  for (int i = 1; i < TERMS; ++i) {
    const unsigned int b = __float_as_uint(rest);
    t[i] = (unsigned short)(b >> 16);
    rest -= __uint_as_float(b & 0xffff0000u);
  }
}

}  // namespace dla
