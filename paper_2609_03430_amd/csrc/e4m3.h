// Rows of an 8-bit cache: 128 OCP E4M3 codes and one power of two per row.
//
// With amax = f * 2^e (1 <= f < 2) the largest |x_c| of a row, the row's
// exponent is s = e - 8 where f <= 1.75 and e - 7 above, so that amax / 2^s lies
// in (224, 448], 448 being the largest code; s >= -126.  code_c = E4M3(x_c /
// 2^s), to nearest even.  An infinite x_c counts as the largest bf16 number, a NaN
// stays one and has no part in the scale.  Where s = 120 the codes end at 240, as
// 256 * 2^120 is past the largest bf16 number.  The scale is held as the byte
// s + 127, in [1, 247].
// A power of two costs an E4M3 row no precision (the codes are floating-point
// themselves, relative step 2^-3 down to amax * 2^-15) and makes the rows
// exact to handle: x / 2^s and code * 2^s need no rounding, a row's value is a
// bf16 number, and writing back what was read gives the same values.
//
// Pools of pool_rows rows: [pool_rows][128] codes, then [pool_rows] scale bytes.
// Key codes are row-major, value codes in tiles of 8 rows stored transposed
// ([row / 8][128][8]), as in the other caches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ra_internal.h"

namespace ra {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Exchanges within rows of 16 lanes that bring every lane together with the others:
// neighbours, pairs, quads (mirrored) and eights (mirrored).
template <typename F>
__device__ __forceinline__ uint32_t over_row16(uint32_t x, F&& join) {
#define RA_DPP(ctrl) \
  static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), ctrl, 0xf, 0xf, false))
  x = join(x, RA_DPP(0xB1));    // quad_perm [1, 0, 3, 2]
  x = join(x, RA_DPP(0x4E));    // quad_perm [2, 3, 0, 1]
  x = join(x, RA_DPP(0x141));   // row_half_mirror
  return join(x, RA_DPP(0x140));   // row_mirror
#undef RA_DPP
}
__device__ __forceinline__ uint32_t max_over_row16(uint32_t x) {
  return over_row16(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// The largest of the lanes with the same lane & 15, in registers: the two rows of 16
// lanes of each half exchanged, then the halves.
__device__ __forceinline__ float max_over_groups(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t m = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ uint32_t max_over_groups(uint32_t u) {
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t m = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return max(b[0], b[1]);
}

// |x| as the scale sees it (its bits).
__device__ __forceinline__ uint32_t row_magnitude(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b > 0x7f800000u ? 0u : min(b, 0x7f7f0000u);
}

// The scale byte of a row whose largest finite magnitude has these bits: the sum
// carries into the exponent where f > 1.75 (bf16 rows never reach byte 248).
__device__ __forceinline__ uint32_t e4m3_scale_byte(uint32_t amax_bits) {
  const int s = static_cast<int>((amax_bits + 0x1fffffu) >> 23) - 8;
  return static_cast<uint32_t>(s < 1 ? 1 : s);
}

__device__ __forceinline__ float e4m3_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float e4m3_inverse(uint32_t byte) {
  return __uint_as_float((254u - byte) << 23);
}

// y within +-limit (comparisons that a NaN fails, so that it stays one).
__device__ __forceinline__ float within(float y, float limit) {
  y = y > limit ? limit : y;
  return y < -limit ? -limit : y;
}

// x divided by the row's scale, within the codes' range.
__device__ __forceinline__ float e4m3_clamp(float y, uint32_t byte) {
  return within(y, byte < 247u ? 448.f : 240.f);
}

// The codes of x and y (divided by the scale and clamped) in the low 16 bits of the
// result, or with HIGH in the high ones, the others taken from `other`.
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_pack2(float x, float y, uint32_t other) {
  return static_cast<uint32_t>(
      __builtin_amdgcn_cvt_pk_fp8_f32(x, y, static_cast<int>(other), HIGH));
}

// Two codes of a word (the low or the high ones) as floats.
template <bool HIGH>
__device__ __forceinline__ f32x2 e4m3_unpack2(uint32_t w) {
  return __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), HIGH);
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Two floats that are bf16 numbers, packed.
__device__ __forceinline__ uint32_t bf16_pack_exact(float lo, float hi) {
  return __float_as_uint(lo) >> 16 | (__float_as_uint(hi) & 0xffff0000u);
}

}  // namespace ra
