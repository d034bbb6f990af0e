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
  // (lanes turned by 8, 4, 2 and 1 within their row of 16)
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x128, 0xf, 0xf, true));
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x124, 0xf, 0xf, true));
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x122, 0xf, 0xf, true));
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x121, 0xf, 0xf, true));
  return m;
}

// m / 127, correctly rounded: the quotient by the rounded 1 / 127 and a correction
// from its exact remainder (checked against the division for every m down to 2^-126).
__device__ __forceinline__ float act8_scale(float m) {
  constexpr float r127 = 1.0f / 127.0f;
  const float q = m * r127;
  return __builtin_fmaf(__builtin_fmaf(-127.0f, q, m), r127, q);
}

// The low bytes of four words.
__device__ __forceinline__ uint32_t act8_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
  return lo | hi << 16;
}

// The codes of this lane's 8 values (bf16 values as floats) and the group's scale, the same
// in all 16 lanes.  The scale of a group with a value that is not finite is NaN.
// A code is the low byte of x (127 / m) + 1.5 2^23, whose last place is 1: one fma
// rounds it, and with the quotient a little too large halves go away from zero.
__device__ __forceinline__ uint2 act8_encode(BF16, const float *x, float *scale) {
  const uint32_t mb = act8_absmax(x);
  const float m = __builtin_bit_cast(float, mb);
  const bool finite = mb < 0x7f800000u, any = finite && mb != 0;
  constexpr float num = 127.0f * (1.0f + 0x1p-19f);  // (the reciprocal's error, 2^-23, is below the 2^-19)
  constexpr uint32_t small = 0x08000000u, large = 0x7d800000u;  // 2^-111, 2^124
  float inv = num * __builtin_amdgcn_rcpf(m), s = act8_scale(m), up = 1.0f;
  if (__builtin_expect(__any(mb < small || mb > large), 0)) {
    // (where 127 / m overflows or 1 / m is below the normal numbers, a power of two goes to x)
    if (mb < small) up = 0x1p60f;
    if (mb > large) up = 0x1p-20f;
    inv = num * __builtin_amdgcn_rcpf(m * up);
    s = m / 127.0f;
  }
  uint32_t c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = __builtin_bit_cast(uint32_t, __builtin_fmaf(x[e] * up, inv, 0x1.8p23f));
  *scale = finite ? s : __builtin_nanf("");
  return any ? make_uint2(act8_bytes(c[0], c[1], c[2], c[3]), act8_bytes(c[4], c[5], c[6], c[7])) : make_uint2(0u, 0u);
}
__device__ __forceinline__ uint2 act8_encode(F32, const float *x, float *scale) {
  const uint32_t mb = act8_absmax(x);
  const float m = __builtin_bit_cast(float, mb);
  const bool finite = mb < 0x7f800000u, any = finite && mb != 0;
  const double inv = 127.0 / (double)m * (1.0 + 0x1p-40);
  uint32_t c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = (uint32_t)__builtin_bit_cast(uint64_t, __builtin_fma((double)x[e], inv, 0x1.8p52));
  *scale = finite ? m / 127.0f : __builtin_nanf("");
  return any ? make_uint2(act8_bytes(c[0], c[1], c[2], c[3]), act8_bytes(c[4], c[5], c[6], c[7])) : make_uint2(0u, 0u);
}

// 8 codes as floats.
__device__ __forceinline__ void act8_floats(uint2 q, float *f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = (float)(int8_t)(q.x >> (8 * e));
    f[4 + e] = (float)(int8_t)(q.y >> (8 * e));
  }
}

// 8 values of type E as loaded, and as floats.
template <class E>
struct Raw8 {
  static constexpr int N = 8 / E::VEC;
  u32x4 v[N];
  template <class I>
  __device__ __forceinline__ void load(const void *base, I i) {
    const typename E::T *p = (const typename E::T *)base + i;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = ld16(p + k * E::VEC);
  }
  // Past the caches: for what is read once, which else takes the place of what comes to be read.
  template <class I>
  __device__ __forceinline__ void load_once(const void *base, I i) {
    const typename E::T *p = (const typename E::T *)base + i;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = __builtin_nontemporal_load((const u32x4 *)(p + k * E::VEC));
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = zero16();
  }
  __device__ __forceinline__ void keep_if(bool in) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = in ? v[k] : zero16();
  }
  __device__ __forceinline__ void get(float *f) const {
#pragma unroll
    for (int k = 0; k < N; ++k) unpack_vec(E(), v[k], f + k * E::VEC);
  }
};
template <class E>
__device__ __forceinline__ void store8(E, void *p, const float *f) {
#pragma unroll
  for (int k = 0; k < 8 / E::VEC; ++k) st16((typename E::T *)p + k * E::VEC, pack_vec(E(), f + k * E::VEC));
}

}  // namespace lora
