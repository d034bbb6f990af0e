// act8.hpp -- activations kept in 8 bits: the codes of a group of 128
// consecutive values of a row, which 16 lanes hold 8 each.
//   m = max |x|,  scale = m / 127,  code = sign(x) floor(127 |x| / m + 1/2)
// so a restored value is off by half a scale at most.  Codes are exact: halves
// are common (x = m / 2 is one), and 127 / m rounds, so the quotient is taken a
// little too large, by less than the distance of any other quotient from the half
// below it.  bf16 values: with x = a 2^i, m = b 2^j, a, b < 2^8, the relative distance
// is 1 / (254 a) at least, 2^-16, and the quotient's is 2^-19.  fp32 values: a, b <
// 2^24, 2^-32 against 2^-40, in 64-bit arithmetic.
#pragma once

#include "kernels.hpp"

namespace lora {

constexpr int ACT8_G = 128;

// Maximum of |x| over the 16 lanes of a group, as bits: these order as the
// values do, and a NaN is above an infinity.
__device__ __forceinline__ uint32_t act8_absmax(const float *x) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __builtin_bit_cast(uint32_t, x[e]) & 0x7fffffffu);
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
  return m;
}

__device__ __forceinline__ uint2 act8_pack(const int *c) {
  uint2 r;
  r.x = (c[0] & 0xff) | (c[1] & 0xff) << 8 | (c[2] & 0xff) << 16 | c[3] << 24;
  r.y = (c[4] & 0xff) | (c[5] & 0xff) << 8 | (c[6] & 0xff) << 16 | c[7] << 24;
  return r;
}

// The codes of this lane's 8 values (bf16 values as floats) and the group's scale, the same
// in all 16 lanes.  The scale of a group with a value that is not finite is NaN.
__device__ __forceinline__ uint2 act8_encode(BF16, const float *x, float *scale) {
  const uint32_t mb = act8_absmax(x);
  const float m = __builtin_bit_cast(float, mb);
  const bool finite = mb < 0x7f800000u, any = finite && mb != 0;
  // (values below 2^-60 are raised by 2^80 first, where 127 / m would overflow)
  const float up = m < 0x1p-60f ? 0x1p80f : 1.0f;
  const float inv = any ? 127.0f / (m * up) * (1.0f + 0x1p-19f) : 0.0f;
  int c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = any ? (int)__builtin_fmaf(x[e] * up, inv, __builtin_copysignf(0.5f, x[e])) : 0;
  *scale = finite ? m / 127.0f : __builtin_nanf("");
  return act8_pack(c);
}
__device__ __forceinline__ uint2 act8_encode(F32, const float *x, float *scale) {
  const uint32_t mb = act8_absmax(x);
  const float m = __builtin_bit_cast(float, mb);
  const bool finite = mb < 0x7f800000u, any = finite && mb != 0;
  const double inv = any ? 127.0 / (double)m * (1.0 + 0x1p-40) : 0.0;
  int c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = any ? (int)__builtin_fma((double)x[e], inv, __builtin_copysign(0.5, (double)x[e])) : 0;
  *scale = finite ? m / 127.0f : __builtin_nanf("");
  return act8_pack(c);
}

// 8 codes as floats.
__device__ __forceinline__ void act8_floats(uint2 q, float *f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = (float)(int8_t)(q.x >> (8 * e));
    f[4 + e] = (float)(int8_t)(q.y >> (8 * e));
  }
}

// 8 values of type E (two vectors in fp32) at p.
__device__ __forceinline__ void load8(BF16, const void *p, float *f) { unpack_vec(BF16(), ld16(p), f); }
__device__ __forceinline__ void load8(F32, const void *p, float *f) {
  unpack_vec(F32(), ld16(p), f);
  unpack_vec(F32(), ld16((const char *)p + 16), f + 4);
}
__device__ __forceinline__ void store8(BF16, void *p, const float *f) { st16(p, pack_vec(BF16(), f)); }
__device__ __forceinline__ void store8(F32, void *p, const float *f) {
  st16(p, pack_vec(F32(), f));
  st16((char *)p + 16, pack_vec(F32(), f + 4));
}

}  // namespace lora
