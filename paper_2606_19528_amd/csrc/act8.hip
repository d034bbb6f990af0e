// act8.hip -- activations to 8 bits and back (act8.hpp): 3 bytes a value in bf16,
// both ways, and nothing else.
#include <algorithm>

#include "act8.hpp"
#include "launch.hpp"

namespace lora {

constexpr int A8_NT = 256, A8_UNITS = A8_NT / 16;  // groups a workgroup holds at a time

// Row and group of unit u < 2^31 with n groups a row: u / n by a multiplication (n > 1).
struct A8Div {
  uint32_t n, mul;
  int shift;
};
static A8Div a8_div(uint32_t n) {
  int l = 0;
  while ((1u << l) < n) ++l;
  const uint64_t one = (uint64_t)1 << (31 + l);
  return A8Div{n, (uint32_t)((one + n - 1) / n), l - 1};
}
__device__ __forceinline__ uint32_t a8_row(const A8Div &d, uint32_t u) {
  return d.n == 1 ? u : __umulhi(u, d.mul) >> d.shift;
}

// What a lane takes of unit u: where its 8 values are, and whether they are there at all.  (Lanes
// without any load the first values: a load in a branch is waited for at its end, so
// the units' loads would come one after the other.)
struct A8At {
  int64_t at;
  bool in;
};
__device__ __forceinline__ A8At a8_at(const A8Div &d, uint32_t u, uint32_t units, int D, int lane) {
  const uint32_t row = a8_row(d, u);
  const int col = (int)(u - row * d.n) * ACT8_G + lane * 8;
  const bool in = u < units && col < D;
  return {in ? (int64_t)row * D + col : 0, in};
}

template <class E, int U>
__global__ __launch_bounds__(A8_NT) void act8_quantize_kernel(const void *x, int8_t *codes, float *scale, uint32_t units, int D,
                                                              A8Div div) {
  const int lane = threadIdx.x & 15;
  const uint32_t u0 = blockIdx.x * (uint32_t)(A8_UNITS * U) + threadIdx.x / 16;
  Raw8<E> r[U];
  A8At a[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    a[k] = a8_at(div, u0 + k * A8_UNITS, units, D, lane);
    if constexpr (U > 1) r[k].load_once(x, a[k].at);
    else r[k].load(x, a[k].at);
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    float f[8], s;
    r[k].keep_if(a[k].in);
    r[k].get(f);
    const uint2 q = act8_encode(E(), f, &s);
    const uint32_t u = u0 + k * A8_UNITS;
    if (a[k].in) *(uint2 *)(codes + a[k].at) = q;
    if (lane == 0 && u < units) scale[u] = s;
  }
}

template <class E, int U>
__global__ __launch_bounds__(A8_NT) void act8_dequantize_kernel(const int8_t *codes, const float *scale, void *x, uint32_t units,
                                                                int D, A8Div div) {
  const int lane = threadIdx.x & 15;
  const uint32_t u0 = blockIdx.x * (uint32_t)(A8_UNITS * U) + threadIdx.x / 16;
  uint2 q[U];
  float s[U];
  A8At a[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const uint32_t u = u0 + k * A8_UNITS;
    a[k] = a8_at(div, u, units, D, lane);
    q[k] = *(const uint2 *)(codes + a[k].at);
    s[k] = scale[u < units ? u : 0];
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    float f[8];
    act8_floats(q[k], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= s[k];
    if (a[k].in) store8(E(), (typename E::T *)x + a[k].at, f);
  }
}

// Few groups: one a 16 lanes, so that more workgroups share them.  Where there are more x is read past the
// caches, which the codes and what comes next then have (4096 x 8192 bf16 18.7 us for 24.9;
// few groups, 1891 x 1000 fp32, 4.3 for 3.6, so not there).
static bool a8_few(int64_t units) { return units < 4 * 256 * A8_UNITS; }

hipError_t launch_act8_quantize(const void *x, int8_t *codes, float *scale, int64_t T, int64_t D, Dtype d, hipStream_t st) {
  const int64_t ng = (D + ACT8_G - 1) / ACT8_G, units = T * ng;
  const A8Div div = a8_div((uint32_t)ng);
  const int u = a8_few(units) ? 1 : 4;
  const dim3 grid((unsigned)((units + A8_UNITS * u - 1) / (A8_UNITS * u))), block(A8_NT);
#define QUANT(E, U) hipLaunchKernelGGL((act8_quantize_kernel<E, U>), grid, block, 0, st, x, codes, scale, (uint32_t)units, (int)D, div)
  if (d == DT_BF16) {
    if (u == 1) QUANT(BF16, 1);
    else QUANT(BF16, 4);
  } else {
    if (u == 1) QUANT(F32, 1);
    else QUANT(F32, 4);
  }
#undef QUANT
  return hipGetLastError();
}

hipError_t launch_act8_dequantize(const int8_t *codes, const float *scale, void *x, int64_t T, int64_t D, Dtype d, hipStream_t st) {
  const int64_t ng = (D + ACT8_G - 1) / ACT8_G, units = T * ng;
  const A8Div div = a8_div((uint32_t)ng);
  const int u = a8_few(units) ? 1 : 4;
  const dim3 grid((unsigned)((units + A8_UNITS * u - 1) / (A8_UNITS * u))), block(A8_NT);
#define DEQUANT(E, U) \
  hipLaunchKernelGGL((act8_dequantize_kernel<E, U>), grid, block, 0, st, codes, scale, x, (uint32_t)units, (int)D, div)
  if (d == DT_BF16) {
    if (u == 1) DEQUANT(BF16, 1);
    else DEQUANT(BF16, 4);
  } else {
    if (u == 1) DEQUANT(F32, 1);
    else DEQUANT(F32, 4);
  }
#undef DEQUANT
  return hipGetLastError();
}

}  // namespace lora
