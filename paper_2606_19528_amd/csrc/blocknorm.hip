// blocknorm.hip -- what stands between two blocks of a decoder, forward: the norm
// behind a block, its gate, the residual scale and sum, and the norm before the next.
//   yn = y r2 (w2 + o)      r2 = 1 / sqrt(mean y^2 + eps)      (yn = y without this norm)
//   h' = h + a g yn
//   n  = h' r1 (w1 + o)     r1 = 1 / sqrt(mean h'^2 + eps)
// One pass over the data (blocknorm.hpp), which the memory path bounds, sums in a fixed order.
// What is stored in fp32 is formed in 64 bits and rounded once: a copy in 8 bits of a value near the middle of
// two codes shows the last bit of it (where h' and n came from products in 32 bits, 103 of 213 million codes were not those of
// the exact values, up to 8e-5 of a copy's norm; now none).  Rows of bf16 values are formed in 32 bits.  8192 x
// 2048 with an fp32 stream 4.85 TB/s, all fp32 4.9 (in 32 bits 5.0 and 4.9).
#include <type_traits>

#include "blocknorm.hpp"

namespace lora {

// 1 / sqrt(mean x^2 + eps) of a row, in 64 bits (F double), or in 32, where rows whose squares leave these are
// summed again in 64 (the branch is the same in all waves of a row, which are a workgroup where
// several).
template <class F, class X, int NV, class S>
__device__ __forceinline__ F row_rstd(const X (&x)[NV][8], int D, double eps, S &sum) {
  if constexpr (std::is_same<F, float>::value) {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = __builtin_fmaf(x[v][e], x[v][e], s);
    s = sum(s);
    if (__builtin_expect(s < __builtin_inff(), 1)) return 1.0f / __builtin_sqrtf(s / (float)D + (float)eps);
  }
  double t = 0.0;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) t = __builtin_fma((double)x[v][e], (double)x[v][e], t);
  t = sum(t);
  return (F)(1.0 / __builtin_sqrt(t / D + eps));
}

// A row's 8 values in 8 bits too, where asked for.  (f: as they are stored.)
template <class E>
__device__ __forceinline__ void keep8(E, const Act8Out &o, const float *f, int64_t row, int D, int ng, int col) {
  float s;
  const uint2 q = act8_encode(E(), f, &s);
  if (col >= D) return;
  *(uint2 *)(o.codes + row * D + (uint32_t)col) = q;
  if (col % ACT8_G == 0) (o.scale + row * ng)[(uint32_t)col / ACT8_G] = s;
}
template <class E>
__device__ __forceinline__ void round_to(E, float *f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = E::to_float(E::from_float(f[e]));
}

__device__ __forceinline__ float bn_fma(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double bn_fma(double a, double b, double c) { return __builtin_fma(a, b, c); }

// ONCE: y and h are read past the caches.
template <class E, class R, int W, int NV, bool ONCE>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void block_norm_fwd_kernel(BlockNormFwd a) {
  constexpr int RPW = W == 1 ? 4 : 1;  // rows of a workgroup
  constexpr bool WIDE = std::is_same<R, F32>::value;
  using H = std::conditional_t<WIDE, double, float>;                         // h' and what goes into it
  using N = std::conditional_t<std::is_same<E, F32>::value, double, float>;  // n
  __shared__ double red[2 * W];
  RowSum<W, W> sum(red);
  const BnCols<W, NV> c{(int)threadIdx.x % (64 * W), a.D};
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * RPW + bn_sub<W>();
  if (row >= a.T) return;  // (a wave's row is its own, or the workgroup's: none waits at a barrier)
  const int D = a.D;
  const int64_t at = row * D;
  const bool each = a.gate_mode == BN_GATE_FULL || a.gate_mode == BN_GATE_CHANNEL;
  Raw8<R> hr[NV];
  Raw8<E> yr[NV], gr[NV], w2[NV], w1[NV];
  // (what is not there is loaded from h instead and not used: the loads stay free of branches)
  bn_load<E, ONCE>(yr, a.y ? a.y : a.h, at, c);
  bn_load<R, ONCE>(hr, a.h, at, c);
  if (each) bn_load<E>(gr, a.gate, a.gate_mode == BN_GATE_FULL ? at : 0, c);
  if (a.w_post) bn_load<E>(w2, a.w_post, 0, c);
  if (a.w_pre) bn_load<E>(w1, a.w_pre, 0, c);
  const float gt = a.gate_mode == BN_GATE_TOKEN ? E::to_float(((const typename E::T *)a.gate)[row]) : 1.0f;
  N x[NV][8];  // h'
  if (a.y) {
    float y[NV][8];
    bn_floats<E>(y, yr, c);
    // (WIDE: y is made anew from what was loaded for each of its uses, and in 64 bits four values at a time: kept
    // it takes the room of a sixth of the waves)
    auto anew = [&](int v) {
      if constexpr (WIDE) {
#pragma unroll
        for (int k = 0; k < Raw8<E>::N; ++k) asm volatile("" : "+v"(yr[v].v[k]));
        yr[v].get(y[v]);
      }
    };
    if (a.y8.codes) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        keep8(E(), a.y8, y[v], row, D, a.ng, c.col(v));
        anew(v);
      }
    }
    H r2 = 1;
    if (a.post) {
      r2 = row_rstd<H>(y, D, a.eps, sum);
      if (c.t == 0 && a.rstd_post) a.rstd_post[row] = (float)r2;
      if constexpr (!WIDE) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          float w[8];
          bn_gain(w, w2[v], a.w_post, (float)a.off);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[v][e] *= r2 * w[e];
        }
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float g[8], h[8], w[8];
      anew(v);
      w2[v].get(w);
      gr[v].get(g);
      hr[v].keep_if(c.in(v));
      hr[v].get(h);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        H yn = (H)y[v][e];
        if constexpr (WIDE) {
          if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
          yn *= r2 * (a.post && a.w_post ? (H)w[e] + (H)a.off : (H)1);  // (without a post norm times 1)
        }
        x[v][e] = (N)bn_fma((H)a.res_scale, yn * (H)(each ? g[e] : gt), (H)h[e]);
      }
    }
    // (lanes past the row hold its last gains and gate, of which an infinity times 0 is no 0)
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] = c.in(v) ? x[v][e] : (N)0;
  } else {
    float h[NV][8];
    bn_floats<R>(h, hr, c);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] = (N)h[v][e];
  }
  // The norm takes the sum before its rounding to a stream of n's type.
  if (a.h_out) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (float)x[v][e];
      if (c.in(v)) store8(R(), (typename R::T *)a.h_out + at + c.at(v), f);
    }
  }
  if (a.h8.codes) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (float)x[v][e];
      round_to(R(), f);
      keep8(R(), a.h8, f, row, D, a.ng, c.col(v));
    }
  }
  if (!a.n && !a.n8.codes && !a.rstd_pre) return;
  const N r1 = row_rstd<N>(x, D, a.eps, sum);
  if (c.t == 0 && a.rstd_pre) a.rstd_pre[row] = (float)r1;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    N w[8];
    float f[8];
    bn_gain(w, w1[v], a.w_pre, (N)a.off);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)(x[v][e] * (r1 * w[e]));
    if (a.n && c.in(v)) store8(E(), (typename E::T *)a.n + at + c.at(v), f);
    if (a.n8.codes) {
      round_to(E(), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = c.in(v) ? f[e] : 0.0f;
      keep8(E(), a.n8, f, row, D, a.ng, c.col(v));
    }
  }
}

template <class E, class R>
static hipError_t fwd_shapes(const BlockNormFwd &a, hipStream_t st) {
  const BnShape s = bn_shape(a.T, a.D);
  const int64_t groups = s.w == 1 ? (a.T + 3) / 4 : a.T, gy = (groups + BN_GRID_ROWS - 1) / BN_GRID_ROWS;
  const dim3 grid((unsigned)((groups + gy - 1) / gy), (unsigned)gy), block(s.w == 1 ? 256 : 64 * s.w);
  // Many rows that are written in 8 bits too are read past the caches, which what is written then has:
  // 16384 x 2048 with three copies 72.9 us for 80.6.  (Without copies it gains nothing, 48.2 for 48.2, and loses
  // where the caches hold h and y: 4096 x 2048 14.8 for 12.6.)
  const bool once = (a.y8.codes || a.h8.codes || a.n8.codes) && (int64_t)a.T * a.D >= (int64_t)1 << 24;
#define FWD(W, NV) hipLaunchKernelGGL((block_norm_fwd_kernel<E, R, W, NV, false>), grid, block, 0, st, a)
#define FWD_ONCE(W, NV) hipLaunchKernelGGL((block_norm_fwd_kernel<E, R, W, NV, true>), grid, block, 0, st, a)
  if (once) {
    BN_SHAPES(s, FWD_ONCE)
  } else {
    BN_SHAPES(s, FWD)
  }
#undef FWD
#undef FWD_ONCE
  return hipGetLastError();
}

hipError_t launch_block_norm_fwd(const BlockNormFwd &a, Dtype d, Dtype res, hipStream_t st) {
  if (d == DT_F32) return fwd_shapes<F32, F32>(a, st);
  return res == DT_F32 ? fwd_shapes<BF16, F32>(a, st) : fwd_shapes<BF16, BF16>(a, st);
}

}  // namespace lora
