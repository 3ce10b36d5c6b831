// Rings in 8 bits.  A row of D features is D E4M3 numbers (OCP: 4 exponent bits, 3 of the significand, no infinities, largest
// 448) and D/32 scale bytes; byte b of a block of 32 features stands for the factor 2^(b - 127) (E8M0).  The scale is the least
// power of two, from 2^-126 on, with which the largest finite feature of the block is at most 448: the block's largest feature
// keeps its three bits and nothing overflows.  A factor that is a power of two rounds nothing itself: a value is the nearest E4M3
// number (ties to even) times it, off by at most 2^-4 of itself or 2^-10 of 2^(b - 127), and both bf16 and fp32 hold it exactly
// (fp32 all of them, from 2^-135 on; bf16 rounds those below 2^-130 to multiples of 2^-133, its least step).  So the matrix cores
// get it as bf16 without another rounding, and packing what was unpacked gives the unpacked values again: after rounding the
// largest feature is at most 448 and at least 224, and where it is 224 exactly the next smaller factor holds the block's values too.
// Infinities and NaN become NaN (E4M3 has no infinity, and a finite number would hide them); they do not count for the scale.
#pragma once
#include "common.hpp"
#include "mfma.hpp"

namespace rattn {

struct fp8_t { uint8_t b; };   // a packed ring's element
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));

constexpr __host__ __device__ int scale_bytes(int D) { return D / 32; }

// the factor of scale byte `byte` of a word of them
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// |x| where x counts for the scale, else 0
__device__ __forceinline__ float finite_abs(float x) {
  const float a = __builtin_fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// Scale byte of a block whose largest finite |x| is a = 1.m 2^E: E + 127 - 8, one more where 1.m is over 448 / 256 = 1.75
__device__ __forceinline__ uint32_t scale_byte(float a) {
  const int f = (int)((__float_as_uint(a) + 0x1fffffu) >> 23) - 8;
  return (uint32_t)max(f, 1);
}
// two codes in the low (HI: high) half of `old`; `inv`: the inverse factor
template <bool HI> __device__ __forceinline__ int two_codes(float x, float y, float inv, int old) {
  x = __builtin_fabsf(x) < INFINITY ? x * inv : __builtin_nanf("");
  y = __builtin_fabsf(y) < INFINITY ? y * inv : __builtin_nanf("");
  return __builtin_amdgcn_cvt_pk_fp8_f32(x, y, old, HI);
}
__device__ __forceinline__ float inverse_factor(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// the value of one element
__device__ __forceinline__ float unpack_one(uint8_t code, uint8_t scale) {
  return __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * scale_of(scale);
}
// four codes as values in bf16, as two registers, or in fp32
__device__ __forceinline__ void unpack_bf16x4(uint32_t codes, float f, uint32_t& lo, uint32_t& hi) {
  lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, f, false));
  hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, f, true));
}
__device__ __forceinline__ f32x4_t unpack_f32x4(uint32_t codes, float f) {
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, f, true);
  return f32x4_t{a[0], a[1], b[0], b[1]};
}

// A row that lies over a wave (feature d in lane d % 64, register d / 64) as codes and scales: a register's two blocks are the
// wave's halves.
template <int EPL>
__device__ __forceinline__ void pack_row(const float (&x)[EPL], uint8_t* codes, uint8_t* scales, int lane) {
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    const float a = row16_reduce(finite_abs(x[e]), [](float p, float q) { return fmaxf(p, q); });
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(a), false, false);
    const uint32_t s = scale_byte(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
    codes[lane + 64 * e] = (uint8_t)two_codes<false>(x[e], 0.f, inverse_factor(s), 0);
    if ((lane & 31) == 0) scales[2 * e + (lane >> 5)] = (uint8_t)s;
  }
}

}  // namespace rattn
