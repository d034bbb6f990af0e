// blocknorm.hpp -- what the norms' two directions share (blocknorm.hip, blocknorm_bwd.hip):
// W waves hold a row, 8 NV values a lane, between the row's sums and its stores.
#pragma once

#include <type_traits>

#include "act8.hpp"
#include "launch.hpp"

namespace lora {

// The 8 values of a lane's vector v of a row: the columns, and where to load them (lanes past
// the row load its last values, so that no load sits in a branch, and hold zeros).
template <int W, int NV>
struct BnCols {
  int t;  // lane of the row, 0 .. 64 W - 1
  int D;
  __device__ __forceinline__ int col(int v) const { return (v * 64 * W + t) * 8; }
  __device__ __forceinline__ bool in(int v) const { return col(v) < D; }
  __device__ __forceinline__ uint32_t at(int v) const { return (uint32_t)min(col(v), D - 8); }
};
// The row of a wave among its workgroup's, as a scalar: a row's addresses are scalars so, and a lane
// holds its offset in the row alone.
template <int W>
__device__ __forceinline__ int bn_sub() { return __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W)); }

template <class E, bool ONCE = false, int W, int NV>
__device__ __forceinline__ void bn_load(Raw8<E> (&r)[NV], const void *p, int64_t at, const BnCols<W, NV> &c) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (ONCE) r[v].load_once((const typename E::T *)p + at, c.at(v));
    else r[v].load((const typename E::T *)p + at, c.at(v));
  }
}
template <class E, int W, int NV>
__device__ __forceinline__ void bn_floats(float (&x)[NV][8], Raw8<E> (&r)[NV], const BnCols<W, NV> &c) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    r[v].keep_if(c.in(v));
    r[v].get(x[v]);
  }
}
// Gains, loaded where there are any.
template <class F, class E>
__device__ __forceinline__ void bn_gain(F *w, const Raw8<E> &r, bool any, F off) {
  float f[8];
  r.get(f);
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = any ? (F)f[e] + off : (F)1;
}

// Sum of a wave, the same bits in each lane: within rows of 16 lanes in turn, then the four rows.
__device__ __forceinline__ float wave_sum(float x) {
#define BN_DPP(ctrl) x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), ctrl, 0xf, 0xf, true))
  BN_DPP(0x128);  // lanes turned by 8, 4, 2, 1
  BN_DPP(0x124);
  BN_DPP(0x122);
  BN_DPP(0x121);
#undef BN_DPP
  const int b = __builtin_bit_cast(int, x);
  const float r0 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(b, 0)), r1 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(b, 16));
  const float r2 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(b, 32)), r3 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(b, 48));
  return (r0 + r1) + (r2 + r3);
}
__device__ __forceinline__ double wave_sum(double x) {
  auto turned = [](double v, auto ctrl) {  // (a double's halves, moved alike)
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_mov_dpp((int)b, decltype(ctrl)::value, 0xf, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_mov_dpp((int)(b >> 32), decltype(ctrl)::value, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  x += turned(x, std::integral_constant<int, 0x128>());
  x += turned(x, std::integral_constant<int, 0x124>());
  x += turned(x, std::integral_constant<int, 0x122>());
  x += turned(x, std::integral_constant<int, 0x121>());
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  auto row = [b](int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((int)b, lane), hi = __builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  return (row(0) + row(16)) + (row(32) + row(48));
}

// Sums over the W waves of a row, NWV waves in the workgroup.
template <int W, int NWV>
struct RowSum {
  double *red;  // [2][NWV] of the workgroup
  int slot;
  __device__ __forceinline__ explicit RowSum(double *r) : red(r), slot(0) {}
  template <class F>
  __device__ __forceinline__ F operator()(F x) {
    x = wave_sum(x);
    if constexpr (W > 1) {
      // (two slots in turn: whoever writes one again has passed the other's barrier, which
      // every reader of the first has reached)
      F *s = (F *)(red + slot * NWV);
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0) s[wave] = x;
      __syncthreads();
      s += wave / W * W;
      x = s[0];
#pragma unroll
      for (int w = 1; w < W; ++w) x += s[w];
      slot ^= 1;
    }
    return x;
  }
};

// Waves a row and vectors a lane, for a row of D columns.  Throughput: two vectors a lane
// (16384 x 2048 forward with its 8-bit copies, read through the caches, 79.7 us, one vector 81.5, four 88; 4096 x 3072
// backward 28.7, one 38, three 30.7).  Few rows: a lane's chain of loads and sums is the time,
// so more waves share a row (one row of 2048 forward 2.2 us, with two waves 3.1).  The longest rows: 1024 x
// 16384 forward 37.6 us, in 8 waves 38.6, with an fp32 stream (in 32 bits) 50 and 52, 51 in 64 bits.
struct BnShape {
  int w, nv;
};
inline BnShape bn_shape(int64_t T, int64_t D) {
  const int64_t n = (D + 511) / 512;  // vectors of a wave
  if (T * n <= 1024) {
    if (n <= 1) return {1, 1};
    if (n <= 4) return {4, 1};
    if (n <= 8) return {8, 1};
    if (n <= 16) return {8, 2};
  }
  if (n <= 2) return {1, (int)n};
  if (n <= 4) return {2, 2};
  if (n <= 6) return {3, 2};
  if (n <= 8) return {4, 2};
  if (n <= 12) return {6, 2};
  if (n <= 16) return {8, 2};
  if (n <= 24) return {12, 2};
  return {16, 2};
}
// Rows of up to 1024 threads each, one a workgroup, in a grid: a dimension holds fewer than 2^32
// threads, so more rows go into the second one (or, in a kernel that takes rows in turn, come later).
constexpr int64_t BN_GRID_ROWS = (int64_t)1 << 21;
static_assert(BN_GRID_ROWS * 1024 < (int64_t)1 << 32, "a grid's dimension");
#define BN_SHAPES(s, CASE)             \
  switch ((s).w * 8 + (s).nv) {        \
    case 1 * 8 + 1: CASE(1, 1); break; \
    case 1 * 8 + 2: CASE(1, 2); break; \
    case 2 * 8 + 2: CASE(2, 2); break; \
    case 3 * 8 + 2: CASE(3, 2); break; \
    case 4 * 8 + 1: CASE(4, 1); break; \
    case 4 * 8 + 2: CASE(4, 2); break; \
    case 6 * 8 + 2: CASE(6, 2); break; \
    case 8 * 8 + 1: CASE(8, 1); break; \
    case 8 * 8 + 2: CASE(8, 2); break; \
    case 12 * 8 + 2: CASE(12, 2); break; \
    default: CASE(16, 2); break;       \
  }

}  // namespace lora
