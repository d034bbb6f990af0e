// blocknorm.hip -- what stands between two blocks of a decoder: the norm behind a
// block, its gate, the residual scale and sum, and the norm before the next block.
//   yn = y r2 (w2 + o)      r2 = 1 / sqrt(mean y^2 + eps)      (yn = y without this norm)
//   h' = h + a g yn
//   n  = h' r1 (w1 + o)     r1 = 1 / sqrt(mean h'^2 + eps)
// and backward from dn and dh' (the stream's gradient behind the block), with hh = h' r1,
// yh = y r2, e = dn (w1 + o):
//   dh = dh' + r1 (e - hh mean(e hh))                 dw1 = sum over rows of dn hh
//   z = a dh,  dyn = g z,  f = dyn (w2 + o)           dg  = z yn, summed where g is broadcast
//   dy = r2 (f - yh mean(f yh))                       dw2 = sum over rows of dyn yh
// One pass over the data: TPR threads hold a row (8 NV values each) between the sums
// and the stores, which the memory path bounds.  Sums are fp32 in a fixed order.
#include <algorithm>

#include "act8.hpp"
#include "launch.hpp"

namespace lora {

// Sums over the TPR threads of a row, the same bits in each.
template <int TPR>
struct RowSum {
  static constexpr int NWV = TPR / 64;
  double *red;  // [2][NWV] of the workgroup, TPR > 64
  int slot;
  __device__ __forceinline__ explicit RowSum(double *r) : red(r), slot(0) {}
  template <class F>
  __device__ __forceinline__ F operator()(F x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
    if constexpr (TPR > 64) {
      // (two slots in turn: whoever writes one again has passed the other's barrier, which
      // every reader of the first has reached)
      F *s = (F *)(red + slot * NWV);
      if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
      __syncthreads();
      x = s[0];
#pragma unroll
      for (int w = 1; w < NWV; ++w) x += s[w];
      slot ^= 1;
    }
    return x;
  }
};

// 1 / sqrt(mean x^2 + eps) of a row.  Rows whose squares leave fp32 are summed again in 64 bits.
template <int TPR, int NV>
__device__ __forceinline__ float row_rstd(const float (&x)[NV][8], int D, float eps, RowSum<TPR> &sum) {
  float s = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __builtin_fmaf(x[v][e], x[v][e], s);
  s = sum(s);
  if (s < __builtin_inff()) return 1.0f / __builtin_sqrtf(s / (float)D + eps);
  double t = 0.0;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) t = __builtin_fma((double)x[v][e], (double)x[v][e], t);
  t = sum(t);
  return (float)(1.0 / __builtin_sqrt(t / D + (double)eps));
}

// Workgroup of rows of TPR threads: several rows where a wave holds one.
constexpr int bn_threads(int tpr) { return tpr == 64 ? 256 : tpr; }

template <class E>
__device__ __forceinline__ void load8(E, const void *p, int64_t i, float *f) {
  Raw8<E> r;
  r.load(p, i);
  r.get(f);
}
template <class E>
__device__ __forceinline__ void round_to(E, float *f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = E::to_float(E::from_float(f[e]));
}

// A row's 8 values in 8 bits too, where asked for.
template <class E>
__device__ __forceinline__ void keep8(E, const Act8Out &o, const float *f, int64_t row, int D, int ng, int col, bool in) {
  float s;
  const uint2 q = act8_encode(E(), f, &s);
  if (!in) return;
  *(uint2 *)(o.codes + row * D + col) = q;
  if (col % ACT8_G == 0) o.scale[row * ng + col / ACT8_G] = s;
}

template <class E, class R, int TPR, int NV>
__global__ __launch_bounds__(bn_threads(TPR)) void block_norm_fwd_kernel(BlockNormFwd a) {
  constexpr int RPW = bn_threads(TPR) / TPR;
  __shared__ double red[2 * (TPR / 64)];
  RowSum<TPR> sum(red);
  const int t = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
  if (row >= a.T) return;  // (TPR > 64: one row a workgroup, so none waits at a barrier)
  const int D = a.D;
  const int64_t at = row * D;
  Raw8<E> yr[NV], gr[NV];
  Raw8<R> hr[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int col = (v * TPR + t) * 8;
    yr[v].zero();
    hr[v].zero();
    gr[v].zero();
    if (col < D) {
      if (a.y) yr[v].load(a.y, at + col);
      hr[v].load(a.h, at + col);
      if (a.gate_mode == BN_GATE_FULL) gr[v].load(a.gate, at + col);
      else if (a.gate_mode == BN_GATE_CHANNEL) gr[v].load(a.gate, col);
    }
  }
  float x[NV][8];
  if (a.y) {
#pragma unroll
    for (int v = 0; v < NV; ++v) yr[v].get(x[v]);
    if (a.y8.codes) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = (v * TPR + t) * 8;
        keep8(E(), a.y8, x[v], row, D, a.ng, col, col < D);
      }
    }
    if (a.post) {
      const float r2 = row_rstd<TPR, NV>(x, D, a.eps, sum);
      if (t == 0 && a.rstd_post) a.rstd_post[row] = r2;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = (v * TPR + t) * 8;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 1.0f;
        if (a.w_post && col < D) {
          load8(E(), a.w_post, col, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] += a.off;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[v][e] *= r2 * w[e];
      }
    }
    const float gt = a.gate_mode == BN_GATE_TOKEN ? E::to_float(((const typename E::T *)a.gate)[row]) : 1.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float g[8], h[8];
      gr[v].get(g);
      hr[v].get(h);
      const bool each = a.gate_mode == BN_GATE_FULL || a.gate_mode == BN_GATE_CHANNEL;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] = __builtin_fmaf(a.res_scale, x[v][e] * (each ? g[e] : gt), h[e]);
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) hr[v].get(x[v]);
  }
  // The norm takes the sum as it is, before its rounding to the stream's type.
  if (a.h_out || a.h8.codes) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * 8;
      if (a.h_out && col < D) store8(R(), (typename R::T *)a.h_out + at + col, x[v]);
      if (a.h8.codes) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = x[v][e];
        round_to(R(), f);
        keep8(R(), a.h8, f, row, D, a.ng, col, col < D);
      }
    }
  }
  if (!a.n && !a.n8.codes && !a.rstd_pre) return;
  const float r1 = row_rstd<TPR, NV>(x, D, a.eps, sum);
  if (t == 0 && a.rstd_pre) a.rstd_pre[row] = r1;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int col = (v * TPR + t) * 8;
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    if (a.w_pre && col < D) {
      load8(E(), a.w_pre, col, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] += a.off;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[v][e] *= r1 * w[e];
    if (a.n && col < D) store8(E(), (typename E::T *)a.n + at + col, x[v]);
    if (a.n8.codes) {
      round_to(E(), x[v]);  // the copy is one of the stored values
      keep8(E(), a.n8, x[v], row, D, a.ng, col, col < D);
    }
  }
}

// ---- backward ----------------------------------------------------------------------
// 8 values of a row kept whole or in 8 bits, as loaded.
template <class E>
struct Src8 {
  Raw8<E> r;
  __device__ __forceinline__ void load(const void *whole, const Act8In &k, int64_t row, int D, int ng, int col) {
    if (k.codes) {
      const uint2 q = *(const uint2 *)(k.codes + row * D + col);
      r.v[0][0] = q.x;
      r.v[0][1] = q.y;
      r.v[0][2] = __builtin_bit_cast(uint32_t, k.scale[row * ng + col / ACT8_G]);
    } else {
      r.load(whole, row * D + col);
    }
  }
  __device__ __forceinline__ void get(const Act8In &k, float *f) const {
    if (k.codes) {
      act8_floats(make_uint2(r.v[0][0], r.v[0][1]), f);
      const u32x4 q = r.v[0];
      const float s = __builtin_bit_cast(float, (uint32_t)q[2]);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= s;
    } else {
      r.get(f);
    }
  }
};

// GRADS: the gradients that are sums over rows too.  A workgroup then takes rows
// blockIdx.x, blockIdx.x + gridDim.x, ... and leaves its sums of each column in
// part[0..2][workgroup (and row of it)][D]: of w1, w2 and a gate [D].
template <class E, class R, int TPR, int NV, bool GRADS>
__global__ __launch_bounds__(bn_threads(TPR)) void block_norm_bwd_kernel(BlockNormBwd a) {
  constexpr int RPW = bn_threads(TPR) / TPR;
  __shared__ double red[2 * (TPR / 64)];
  RowSum<TPR> sum(red);
  const int t = threadIdx.x % TPR;
  const int D = a.D;
  const float inv_d = 1.0f / (float)D;
  const bool need_y = a.post || a.dgate;
  float s1[NV][8], s2[NV][8], sg[NV][8];
  if constexpr (GRADS) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) s1[v][e] = s2[v][e] = sg[v][e] = 0.0f;
  }
  const int64_t first = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR, step = (int64_t)gridDim.x * RPW;
  for (int64_t row = first; row < a.T; row += step) {
    const int64_t at = row * D;
    Raw8<E> dn[NV], g[NV];
    Raw8<R> dho[NV];
    Src8<R> hs[NV];
    Src8<E> ys[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * 8;
      dn[v].zero();
      g[v].zero();
      dho[v].zero();
      hs[v].r.zero();
      ys[v].r.zero();
      if (col < D) {
        if (a.dn) {
          dn[v].load(a.dn, at + col);
          hs[v].load(a.h, a.h8, row, D, a.ng, col);
        }
        if (a.dh_out) dho[v].load(a.dh_out, at + col);
        if (need_y) ys[v].load(a.y, a.y8, row, D, a.ng, col);
        if (a.gate_mode == BN_GATE_FULL) g[v].load(a.gate, at + col);
        else if (a.gate_mode == BN_GATE_CHANNEL) g[v].load(a.gate, col);
      }
    }
    float dh[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) dho[v].get(dh[v]);
    if (a.dn) {
      const float r1 = a.rstd_pre[row];
      float c = 0.0f;
      float hh[NV][8], ee[NV][8];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = (v * TPR + t) * 8;
        hs[v].get(a.h8, hh[v]);
        dn[v].get(ee[v]);
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          hh[v][e] *= r1;
          w[e] = 1.0f;
        }
        if (a.w_pre && col < D) {
          load8(E(), a.w_pre, col, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] += a.off;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (GRADS) s1[v][e] = __builtin_fmaf(ee[v][e], hh[v][e], s1[v][e]);
          ee[v][e] *= w[e];
          c = __builtin_fmaf(ee[v][e], hh[v][e], c);
        }
      }
      c = sum(c) * inv_d;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) dh[v][e] = __builtin_fmaf(r1, __builtin_fmaf(-hh[v][e], c, ee[v][e]), dh[v][e]);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * 8;
      if (a.dh && col < D) store8(R(), (typename R::T *)a.dh + at + col, dh[v]);
    }
    if (!a.dy && !a.dgate && !a.want_w2) continue;
    // dh becomes f (dyn without this norm), y becomes yh
    float y[NV][8];
    const float r2 = a.post ? a.rstd_post[row] : 1.0f;
    const float gt = a.gate_mode == BN_GATE_TOKEN ? E::to_float(((const typename E::T *)a.gate)[row]) : 1.0f;
    const bool each = a.gate_mode == BN_GATE_FULL || a.gate_mode == BN_GATE_CHANNEL;
    float c2 = 0.0f, dgt = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * 8;
      float w[8], gv[8];
      ys[v].get(a.y8, y[v]);
      g[v].get(gv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[v][e] *= r2;
        w[e] = 1.0f;
      }
      if (a.w_post && col < D) {
        load8(E(), a.w_post, col, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] += a.off;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = a.res_scale * dh[v][e], yw = y[v][e] * w[e];
        dgt = __builtin_fmaf(z, yw, dgt);
        const float dyn = z * (each ? gv[e] : gt);
        if constexpr (GRADS) {
          sg[v][e] = __builtin_fmaf(z, yw, sg[v][e]);
          s2[v][e] = __builtin_fmaf(dyn, y[v][e], s2[v][e]);
        }
        gv[e] = z * yw;
        dh[v][e] = dyn * w[e];
        c2 = __builtin_fmaf(dh[v][e], y[v][e], c2);
      }
      if (a.dgate && a.gate_mode == BN_GATE_FULL && col < D) store8(E(), (typename E::T *)a.dgate + at + col, gv);
    }
    if (a.dgate && a.gate_mode == BN_GATE_TOKEN) {
      dgt = sum(dgt);
      if (t == 0) ((float *)a.dgate)[row] = dgt;
    }
    if (!a.dy) continue;
    if (a.post) c2 = sum(c2) * inv_d;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * 8;
      if (a.post) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dh[v][e] = r2 * __builtin_fmaf(-y[v][e], c2, dh[v][e]);
      }
      if (col < D) store8(E(), (typename E::T *)a.dy + at + col, dh[v]);
    }
  }
  if constexpr (GRADS) {
    const int64_t p = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
    const int64_t plane = (int64_t)gridDim.x * RPW * D;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * 8;
      if (col >= D) continue;
      float *o = a.part + p * D + col;
      if (a.want_w1) store8(F32(), o, s1[v]);
      if (a.want_w2) store8(F32(), o + plane, s2[v]);
      if (a.want_gate) store8(F32(), o + 2 * plane, sg[v]);
    }
  }
}

// out[c] = sum over p < np of part[p][c], ascending in 16 ranges of p: 16 columns a
// workgroup (D of a few thousand then gives hundreds of them).
__global__ __launch_bounds__(256) void block_norm_cols_kernel(const float *part, int np, int D, float *o1, float *o2, float *og) {
  __shared__ float red[16][17];
  const int which = blockIdx.y;
  float *out = which == 0 ? o1 : which == 1 ? o2 : og;
  if (!out) return;
  const int c = threadIdx.x & 15, s = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  const float *src = part + (int64_t)which * np * D;
  const int per = (np + 15) / 16, p1 = min(np, (s + 1) * per);
  float x = 0.0f;
  if (col < D)
    for (int p = s * per; p < p1; ++p) x += src[(int64_t)p * D + col];
  red[s][c] = x;
  __syncthreads();
  if (s == 0 && col < D) {
#pragma unroll
    for (int k = 1; k < 16; ++k) x += red[k][c];
    out[col] = x;
  }
}

// Threads that hold a row of D columns, 8 NV values each, and the rows of a workgroup.
struct BnShape {
  int tpr, nv, rows;
};
static BnShape bn_shape(int64_t D) {
  if (D <= 512) return {64, 1, 4};
  if (D <= 1024) return {64, 2, 4};
  if (D <= 2048) return {128, 2, 1};
  if (D <= 4096) return {256, 2, 1};
  if (D <= 8192) return {512, 2, 1};
  return {1024, 2, 1};
}
constexpr int BN_PARTS = 512;  // workgroups that sum over rows

int block_norm_parts(int64_t T, int64_t D) {
  const BnShape s = bn_shape(D);
  return (int)std::min<int64_t>((T + s.rows - 1) / s.rows, BN_PARTS) * s.rows;
}

#define BN_SIZES(CASE)                                                                                  \
  switch (s.tpr * s.nv) {                                                                               \
    case 64: CASE(64, 1); break;                                                                        \
    case 128: CASE(64, 2); break;                                                                       \
    case 256: CASE(128, 2); break;                                                                      \
    case 512: CASE(256, 2); break;                                                                      \
    case 1024: CASE(512, 2); break;                                                                     \
    default: CASE(1024, 2); break;                                                                      \
  }

template <class E, class R>
static hipError_t fwd_sizes(const BlockNormFwd &a, hipStream_t st) {
  const BnShape s = bn_shape(a.D);
  const dim3 grid((unsigned)((a.T + s.rows - 1) / s.rows));
#define FWD(TPR, NV) hipLaunchKernelGGL((block_norm_fwd_kernel<E, R, TPR, NV>), grid, dim3(bn_threads(TPR)), 0, st, a)
  BN_SIZES(FWD)
#undef FWD
  return hipGetLastError();
}

template <class E, class R>
static hipError_t bwd_sizes(const BlockNormBwd &a, hipStream_t st) {
  const BnShape s = bn_shape(a.D);
  const bool grads = a.want_w1 || a.want_w2 || a.want_gate;
  const int np = block_norm_parts(a.T, a.D);
  const dim3 grid(grads ? (unsigned)(np / s.rows) : (unsigned)((a.T + s.rows - 1) / s.rows));
#define BWD(TPR, NV)                                                                                                      \
  if (grads) hipLaunchKernelGGL((block_norm_bwd_kernel<E, R, TPR, NV, true>), grid, dim3(bn_threads(TPR)), 0, st, a);       \
  else hipLaunchKernelGGL((block_norm_bwd_kernel<E, R, TPR, NV, false>), grid, dim3(bn_threads(TPR)), 0, st, a)
  BN_SIZES(BWD)
#undef BWD
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !grads) return e;
  hipLaunchKernelGGL(block_norm_cols_kernel, dim3((a.D + 15) / 16, 3), dim3(256), 0, st, a.part, np, a.D, a.want_w1, a.want_w2,
                     a.want_gate);
  return hipGetLastError();
}

hipError_t launch_block_norm_fwd(const BlockNormFwd &a, Dtype d, Dtype res, hipStream_t st) {
  if (d == DT_F32) return fwd_sizes<F32, F32>(a, st);
  return res == DT_F32 ? fwd_sizes<BF16, F32>(a, st) : fwd_sizes<BF16, BF16>(a, st);
}
hipError_t launch_block_norm_bwd(const BlockNormBwd &a, Dtype d, Dtype res, hipStream_t st) {
  if (d == DT_F32) return bwd_sizes<F32, F32>(a, st);
  return res == DT_F32 ? bwd_sizes<BF16, F32>(a, st) : bwd_sizes<BF16, BF16>(a, st);
}

}  // namespace lora
