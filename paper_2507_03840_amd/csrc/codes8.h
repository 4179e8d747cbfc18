// 8-bit codes: e4m3 (1 sign, 4 exponent, 3 mantissa bits, largest value 448, no infinities) times a power of two for a block of 128 values.
//
// The scale of a block is 2^e, held as the byte e + 127 (e8m0, as the matrix instructions take it), with e the least integer for which the
// block's largest finite magnitude times 2^-e is at most 448; e >= -127, so a block of zeros has the byte 0.  A power of two costs no accuracy: a
// floating element keeps its relative precision wherever in the range it lies, dividing by the scale is exact, and a code times its scale is
// exact in bfloat16.  One rounding, to nearest even, of value 2^-e to e4m3: at most 2^-4 of the value, or 2^-10 2^e below 2^-6 2^e.
// What is not finite becomes NaN (0x7f), the only code that is neither a number nor zero, and does not count for the scale.
#pragma once
#include "row_types.h"

#define C8_BLOCK 128

inline int c8_blocks(int64_t n) { return (int)((n + C8_BLOCK - 1) / C8_BLOCK); }
inline int64_t c8_round16(int64_t n) { return (n + 15) / 16 * 16; }

// Byte of the scale for a largest magnitude given as the bits of a finite float >= 0: with magnitude m 2^k, 1 <= m < 2, and 448 = 1.75 2^8,
// e is k - 8 up to m = 1.75 and k - 7 above.  (Subnormals have e < -127 and are clamped like zero.)
__device__ __forceinline__ int c8_scale_byte(unsigned largest) {
  const int b = (int)(largest >> 23) - 8 + ((largest & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b > 0 ? b : 0;
}
// 2^-e of a scale byte up to 253 (a float's largest gives 247)
__device__ __forceinline__ float c8_inverse(int byte) { return __uint_as_float((unsigned)(254 - byte) << 23); }

// bits of |v| where v is finite, 0 elsewhere: what counts for the scale
__device__ __forceinline__ unsigned c8_magnitude(float v) {
  const unsigned a = __float_as_uint(v) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}
// value on the scale, NaN for an infinite one (whatever the conversion makes of that)
__device__ __forceinline__ float c8_scaled(float v, float inverse) {
  return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u ? v * inverse : __uint_as_float(0x7fc00000u);
}
// two values to the low half of a word, four to a word
__device__ __forceinline__ unsigned c8_pair(float a, float b) { return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu; }
__device__ __forceinline__ unsigned c8_four(float a, float b, float c, float d) {
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

__device__ __forceinline__ unsigned c8_wave_max(unsigned v, int lanes) {
  for (int at = lanes >> 1; at; at >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, at));
  return v;
}
__device__ __forceinline__ double c8_wave_sum(double v, int lanes) {
  for (int at = lanes >> 1; at; at >>= 1) v += __shfl_xor(v, at);
  return v;
}

// Codes of N x V values of one block, which `lanes` neighbouring lanes hold together (lanes a power of two, the same for all of the wave; a lane without
// values holds zeros): returns the scale byte, v becomes the values on the scale.  What is not finite is looked at apart, where there is any.
template <int N>
__device__ __forceinline__ int c8_to_scale(float (&v)[N], int lanes) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  if (__any(m >= 0x7f800000u)) {
    m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      m = max(m, c8_magnitude(v[i]));
      v[i] = c8_scaled(v[i], 1.0f);
    }
  }
  const int byte = c8_scale_byte(c8_wave_max(m, lanes));
  const float inverse = c8_inverse(byte);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] *= inverse;
  return byte;
}
// V codes to an address of a multiple of V
template <int V>
__device__ __forceinline__ void c8_store(uint8_t* q, const float (&v)[V]) {
  static_assert(V == 4 || V == 8, "a word or two");
  if constexpr (V == 4) *(unsigned*)q = c8_four(v[0], v[1], v[2], v[3]);
  else *(uint2*)q = make_uint2(c8_four(v[0], v[1], v[2], v[3]), c8_four(v[4], v[5], v[6], v[7]));
}

// A block of up to 128 values of one row, two a lane of a whole wave (columns c0 + lane and c0 + 64 + lane of n): codes, zeros up to the next
// multiple of 16 columns behind the last, and the scale.
__device__ __forceinline__ void c8_store_block(float v0, float v1, int c0, int n, int lane, uint8_t* q, uint8_t* scale) {
  const int a = c0 + lane, b = a + 64, end = (n + 15) & ~15;
  const unsigned m0 = a < n ? c8_magnitude(v0) : 0u, m1 = b < n ? c8_magnitude(v1) : 0u;
  const int byte = c8_scale_byte(c8_wave_max(max(m0, m1), 64));
  const float inverse = c8_inverse(byte);
  const unsigned two = c8_pair(c8_scaled(v0, inverse), c8_scaled(v1, inverse));
  if (a < end) q[a] = a < n ? (uint8_t)(two & 0xff) : 0;
  if (b < end) q[b] = b < n ? (uint8_t)(two >> 8) : 0;
  if (lane == 0) *scale = (uint8_t)byte;
}
