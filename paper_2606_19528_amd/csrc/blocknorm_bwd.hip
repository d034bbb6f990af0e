// blocknorm_bwd.hip -- the backward of blocknorm.hip, from dn and dh', the gradients of
// the next block's normed input and of the stream behind this one.  With hh = h' r1, yh = y r2,
// e = dn (w1 + o):
//   dh = dh' + r1 (e - hh mean(e hh))                 dw1 = sum over rows of dn hh
//   z = a dh,  f = g z (w2 + o)                       dg  = z yn, summed where g is broadcast
//   dy = r2 (f - yh mean(f yh))                       dw2 = sum over rows of g z yh
// One pass over the data (blocknorm.hpp): 4096 x 3072 in bf16 from 8-bit copies 25.4 us (126 MB, 5.0
// TB/s), where a form with a branch a vector took 52: beside the memory path the vector
// instructions count, a few hundred for 8 columns.  dh is linear in the
// first mean, so that the second comes from sums taken with it: dh = p - c q with
// p = dh' + r1 e, q = r1 hh and c = mean(e hh), and for weights k of a column
//   sum k dh yh = sum k p yh - c sum k q yh,
// one meeting of a row's waves instead of two.  Sums are fp32 in a fixed order.
#include <algorithm>

#include "blocknorm.hpp"

namespace lora {

// A row kept whole or in 8 bits, as loaded.  (Here and below one branch stands around all of a
// lane's vectors: a branch in each kept the loads from being ahead of one another.)
template <class E, int W, int NV>
__device__ __forceinline__ void src_load(Raw8<E> (&r)[NV], const void *whole, const Act8In &k, int64_t row, int ng,
                                         const BnCols<W, NV> &c) {
  if (k.codes) {
    const int8_t *q = k.codes + row * c.D;
    const float *s = k.scale + row * ng;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const uint2 t = *(const uint2 *)(q + c.at(v));
      r[v].v[0] = u32x4{t.x, t.y, __builtin_bit_cast(uint32_t, s[c.at(v) / ACT8_G]), 0u};
    }
  } else {
    bn_load<E>(r, whole, row * c.D, c);
  }
}
template <class E, int NV>
__device__ __forceinline__ void src_floats(float (&x)[NV][8], const Raw8<E> (&r)[NV], const Act8In &k, float m) {
  if (k.codes) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const u32x4 q = r[v].v[0];
      act8_floats(make_uint2(q[0], q[1]), x[v]);
      const float s = __builtin_bit_cast(float, (uint32_t)q[2]) * m;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= s;
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      r[v].get(x[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= m;
    }
  }
}
// x *= gains + off.
template <class E, int NV>
__device__ __forceinline__ void times(float (&x)[NV][8], const Raw8<E> (&w)[NV], float off) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    float f[8];
    w[v].get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[v][e] *= f[e] + off;
  }
}

// GRADS: the gradients that are sums over rows too.  Workgroups of bnb_waves waves then, which take rows in
// turn and leave their sums of each column in part[0..1][workgroup][D]: of dn hh, and of a yh dh times
// the gate where that has a value a row; the sums for w2 and for a gate [D] are this one times the
// column's gate or gain.
constexpr int bnb_waves(int w, bool wide) { return w > 12 ? w : w % 3 == 0 || (!wide && w > 1 && w < 8) ? 12 : 8; }
constexpr int bnb_rows(int w, bool grads, bool wide) { return grads ? bnb_waves(w, wide) / w : w == 1 ? 4 : 1; }
constexpr int bnb_threads(int w, bool grads, bool wide) { return 64 * w * bnb_rows(w, grads, wide); }

// ONCE: dn and dh' are read past the caches.
template <class E, class R, int W, int NV, bool GRADS, bool ONCE>
__global__ __launch_bounds__(bnb_threads(W, GRADS, R::VEC == 4)) void block_norm_bwd_kernel(BlockNormBwd a) {
  constexpr int RPW = bnb_rows(W, GRADS, R::VEC == 4), NWV = W * RPW;  // rows and waves of a workgroup
  __shared__ float red[2][3][NWV];
  const BnCols<W, NV> c{(int)threadIdx.x % (64 * W), a.D};
  const int D = a.D, sub = bn_sub<W>(), wave = threadIdx.x >> 6;
  const float inv_d = 1.0f / (float)D;
  const bool need_y = a.post || a.dgate, block = a.dy || a.dgate || a.want_w2;
  float s1[NV][8], sz[NV][8];
  if constexpr (GRADS) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) s1[v][e] = sz[v][e] = 0.0f;
  }
  int slot = 0;
  Raw8<E> w1[NV], w2[NV];  // (the same for all rows)
  if (a.w_pre) bn_load<E>(w1, a.w_pre, 0, c);
  if (a.w_post) bn_load<E>(w2, a.w_post, 0, c);
  // (all waves of a workgroup go round as often as its first row needs)
  for (int64_t r0 = (int64_t)blockIdx.x * RPW; r0 < a.T; r0 += (int64_t)gridDim.x * RPW) {
    const bool live = r0 + sub < a.T;
    const int64_t row = live ? r0 + sub : a.T - 1, at = row * D;
    Raw8<E> dnr[NV], yr[NV], gr[NV];
    Raw8<R> dhr[NV], hr[NV];
    if (a.dn) {
      bn_load<E, ONCE>(dnr, a.dn, at, c);
      src_load<R>(hr, a.h, a.h8, row, a.ng, c);
    }
    if (a.dh_out) bn_load<R, ONCE>(dhr, a.dh_out, at, c);
    if (need_y) src_load<E>(yr, a.y, a.y8, row, a.ng, c);
    if (a.gate_mode & 1) bn_load<E>(gr, a.gate, a.gate_mode == BN_GATE_FULL ? at : 0, c);  // (channel, full)
    const float r1 = a.dn ? a.rstd_pre[row] : 0.0f, r2 = a.post ? a.rstd_post[row] : 1.0f;
    const float gt = a.gate_mode == BN_GATE_TOKEN ? E::to_float(((const typename E::T *)a.gate)[row]) : 1.0f;
    float h[NV][8], p[NV][8], y[NV][8], k[NV][8];  // hh, p and then dh, yh
    float ca = 0.0f, cb = 0.0f, cc = 0.0f;
    // e = dn (w1 + o), p = dh' + r1 e.  Lanes past the row, and rows past the last, have dn, dh' and y
    // zeros, so that they add nothing to a sum.
    if (a.dn) {
      src_floats<R>(h, hr, a.h8, r1);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        dnr[v].keep_if(live && c.in(v));
        dnr[v].get(p[v]);
        if constexpr (GRADS) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s1[v][e] = __builtin_fmaf(p[v][e], h[v][e], s1[v][e]);
        }
      }
      if (a.w_pre) times<E>(p, w1, a.off);
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ca = __builtin_fmaf(p[v][e], h[v][e], ca);
          p[v][e] *= r1;
        }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) h[v][e] = p[v][e] = 0.0f;
    }
    if (a.dh_out) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float f[8];
        dhr[v].keep_if(live && c.in(v));  // (an infinity there times y's zeros would be a NaN in a sum)
        dhr[v].get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[v][e] += f[e];
      }
    }
    // k = a g (w2 + o), without a gate a token: f = k gt dh
    if (block) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) k[v][e] = a.res_scale;
      if (a.gate_mode & 1) times<E>(k, gr, 0.0f);
      if (a.w_post) times<E>(k, w2, a.off);
      if (need_y) {
#pragma unroll
        for (int v = 0; v < NV; ++v) yr[v].keep_if(live && c.in(v));
        src_floats<E>(y, yr, a.y8, r2);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float ky = k[v][e] * y[v][e];
            cb = __builtin_fmaf(ky, p[v][e], cb);
            cc = __builtin_fmaf(ky, h[v][e], cc);
          }
      }
    }
    ca = wave_sum(ca);
    cb = wave_sum(cb);
    cc = wave_sum(cc);
    if constexpr (W > 1) {
      // (two slots in turn: whoever writes one again has passed the other's barrier, which
      // every reader of the first has reached)
      float(*s)[NWV] = red[slot];
      if ((threadIdx.x & 63) == 0) {
        s[0][wave] = ca;
        s[1][wave] = cb;
        s[2][wave] = cc;
      }
      __syncthreads();
      const int w0 = sub * W;
      ca = s[0][w0];
      cb = s[1][w0];
      cc = s[2][w0];
#pragma unroll
      for (int w = 1; w < W; ++w) {
        ca += s[0][w0 + w];
        cb += s[1][w0 + w];
        cc += s[2][w0 + w];
      }
      slot ^= 1;
    }
    const float q = r1 * (ca * inv_d);            // dh = p - q hh
    const float fy = __builtin_fmaf(-q, cc, cb);  // sum k dh yh
    if (a.gate_mode == BN_GATE_TOKEN && a.dgate && c.t == 0 && live) ((float *)a.dgate)[row] = fy;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[v][e] = __builtin_fmaf(-q, h[v][e], p[v][e]);
      if (live && c.in(v)) store8(R(), (typename R::T *)a.dh + at + c.at(v), p[v]);
    }
    if (!block) continue;
    if constexpr (GRADS) {
      if (a.want_w2 || a.want_gate) {
        if (a.gate_mode == BN_GATE_FULL) {
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            float g[8];
            gr[v].get(g);
#pragma unroll
            for (int e = 0; e < 8; ++e) sz[v][e] = __builtin_fmaf(a.res_scale * y[v][e] * p[v][e], g[e], sz[v][e]);
          }
        } else {
          const float m = a.res_scale * gt;
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) sz[v][e] = __builtin_fmaf(m * y[v][e], p[v][e], sz[v][e]);
        }
      }
    }
    if (a.dgate && a.gate_mode == BN_GATE_FULL) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) h[v][e] = a.res_scale * y[v][e] * p[v][e];
      if (a.w_post) times<E>(h, w2, a.off);
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (live && c.in(v)) store8(E(), (typename E::T *)a.dgate + at + c.at(v), h[v]);
    }
    if (!a.dy) continue;
    // dy = r2 (f - yh mean(f yh)), or f
    const float kf = gt * r2, c2 = kf * (fy * inv_d);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[v][e] = k[v][e] * kf * p[v][e];
      if (a.post) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[v][e] = __builtin_fmaf(-c2, y[v][e], p[v][e]);
      }
      if (live && c.in(v)) store8(E(), (typename E::T *)a.dy + at + c.at(v), p[v]);
    }
  }
  if constexpr (GRADS) {
    // The rows' sums of the workgroup, one array after the other.
    __shared__ float cols[RPW > 1 ? RPW - 1 : 1][64 * W * NV * 8 + 4];
    const int64_t plane = (int64_t)gridDim.x * D;
    float *const out = a.part + (int64_t)blockIdx.x * D;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (!(which == 0 ? a.want_w1 : a.want_w2 ? a.want_w2 : a.want_gate)) continue;
      float(&s)[NV][8] = which == 0 ? s1 : sz;
      if constexpr (RPW > 1) {
        __syncthreads();
        if (sub > 0) {
#pragma unroll
          for (int v = 0; v < NV; ++v) store8(F32(), &cols[sub - 1][c.col(v)], s[v]);
        }
        __syncthreads();
      }
      if (sub == 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
          for (int k = 1; k < RPW; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[v][e] += cols[k - 1][c.col(v) + e];
          if (c.in(v)) store8(F32(), out + which * plane + c.col(v), s[v]);
        }
      }
    }
  }
}

// Rows whose values do not fit a workgroup's registers (over 12288 columns, or 8192 with a stream of fp32 or sums over
// rows): 16 waves (up to 12288 columns 12, fp32 8, which leave the registers for it) take two passes over a row, the first
// for the three sums, the second for the outputs, a vector of a lane after the other; what the second reads is in
// the caches.  Sums over rows stand in LDS, each lane's its own.  1024 x 16384 bf16 56 us, with sums 59, fp32
// 118; with all of a row in registers, some of which go through memory, 116, 263 and 265.
template <class E, class R>
struct BnbVec {
  Raw8<E> dn[1], y[1], g[1], w1[1], w2[1];
  Raw8<R> dho[1], h[1];
  template <int W>
  __device__ __forceinline__ void load(const BlockNormBwd &a, int64_t row, const BnCols<W, 1> &c, bool need_y) {
    const int64_t at = row * c.D;
    if (a.dn) {
      bn_load<E>(dn, a.dn, at, c);
      src_load<R>(h, a.h, a.h8, row, a.ng, c);
      if (a.w_pre) bn_load<E>(w1, a.w_pre, 0, c);
    }
    if (a.dh_out) bn_load<R>(dho, a.dh_out, at, c);
    if (need_y) src_load<E>(y, a.y, a.y8, row, a.ng, c);
    if (a.gate_mode & 1) bn_load<E>(g, a.gate, a.gate_mode == BN_GATE_FULL ? at : 0, c);
    if (a.w_post) bn_load<E>(w2, a.w_post, 0, c);
  }
  // dn, hh, p, yh and k of the vector (dn, dh' and yh zeros past the row).
  template <int W>
  __device__ __forceinline__ void floats(const BlockNormBwd &a, const BnCols<W, 1> &c, float r1, float r2, bool need_y,
                                         float (&d)[1][8], float (&x)[1][8], float (&p)[1][8], float (&z)[1][8],
                                         float (&k)[1][8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) d[0][e] = x[0][e] = p[0][e] = z[0][e] = 0.0f, k[0][e] = a.res_scale;
    if (a.dn) {
      src_floats<R>(x, h, a.h8, r1);
      dn[0].keep_if(c.in(0));
      dn[0].get(d[0]);
#pragma unroll
      for (int e = 0; e < 8; ++e) p[0][e] = d[0][e];
      if (a.w_pre) times<E>(p, w1, a.off);
    }
    if (a.gate_mode & 1) times<E>(k, g, 0.0f);
    if (a.w_post) times<E>(k, w2, a.off);
    if (need_y) {
      y[0].keep_if(c.in(0));
      src_floats<E>(z, y, a.y8, r2);
    }
    dho[0].keep_if(c.in(0));  // (an infinity there times y's zeros would be a NaN in a sum)
  }
  // p, which is e, becomes dh' + r1 e.
  __device__ __forceinline__ void add_stream(const BlockNormBwd &a, float r1, float (&p)[1][8]) {
    float f[8];
    dho[0].get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) p[0][e] = a.dh_out ? __builtin_fmaf(r1, p[0][e], f[e]) : r1 * p[0][e];
  }
};

template <class E, class R, int W, int NV, bool GRADS>
__global__ __launch_bounds__(64 * W) void block_norm_bwd_long_kernel(BlockNormBwd a) {
  constexpr int NT = 64 * W;
  __shared__ float red[2][3][W];
  __shared__ f32x4 sums[GRADS ? 2 * NV * 2 : 1][GRADS ? NT : 1];  // [which][vector][half][lane]
  const int D = a.D, t = threadIdx.x, wave = t >> 6, nv = (D + 8 * NT - 1) / (8 * NT);
  const float inv_d = 1.0f / (float)D;
  const bool need_y = a.post || a.dgate, block = a.dy || a.dgate || a.want_w2;
  auto cols = [&](int v) { return BnCols<W, 1>{v * NT + t, D}; };
  if constexpr (GRADS) {
#pragma unroll
    for (int k = 0; k < 4 * NV; ++k) sums[k][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  auto add = [&](int k, const float *f) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      f32x4 x = sums[2 * k + half][t];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += f[4 * half + e];
      sums[2 * k + half][t] = x;
    }
  };
  int slot = 0;
  for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    const int64_t at = row * D;
    const float r1 = a.dn ? a.rstd_pre[row] : 0.0f, r2 = a.post ? a.rstd_post[row] : 1.0f;
    const float gt = a.gate_mode == BN_GATE_TOKEN ? E::to_float(((const typename E::T *)a.gate)[row]) : 1.0f;
    float d[1][8], h[1][8], p[1][8], y[1][8], k[1][8];
    float ca = 0.0f, cb = 0.0f, cc = 0.0f;
#pragma unroll 1
    for (int v = 0; v < nv; ++v) {
      BnbVec<E, R> x;
      x.load(a, row, cols(v), need_y);
      x.floats(a, cols(v), r1, r2, need_y, d, h, p, y, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) ca = __builtin_fmaf(p[0][e], h[0][e], ca);
      x.add_stream(a, r1, p);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float ky = k[0][e] * y[0][e];
        cb = __builtin_fmaf(ky, p[0][e], cb);
        cc = __builtin_fmaf(ky, h[0][e], cc);
      }
    }
    ca = wave_sum(ca);
    cb = wave_sum(cb);
    cc = wave_sum(cc);
    // (two slots in turn, as in the kernel above)
    float(*s)[W] = red[slot];
    if ((t & 63) == 0) {
      s[0][wave] = ca;
      s[1][wave] = cb;
      s[2][wave] = cc;
    }
    __syncthreads();
    ca = s[0][0];
    cb = s[1][0];
    cc = s[2][0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      ca += s[0][w];
      cb += s[1][w];
      cc += s[2][w];
    }
    slot ^= 1;
    const float q = r1 * (ca * inv_d);            // dh = p - q hh
    const float fy = __builtin_fmaf(-q, cc, cb);  // sum k dh yh
    if (a.gate_mode == BN_GATE_TOKEN && a.dgate && t == 0) ((float *)a.dgate)[row] = fy;
    const float kf = gt * r2, c2 = kf * (fy * inv_d);
#pragma unroll 1
    for (int v = 0; v < nv; ++v) {
      const BnCols<W, 1> c = cols(v);
      BnbVec<E, R> x;
      x.load(a, row, c, need_y);
      x.floats(a, c, r1, r2, need_y, d, h, p, y, k);
      x.add_stream(a, r1, p);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[0][e] = __builtin_fmaf(-q, h[0][e], p[0][e]);
        d[0][e] *= h[0][e];
      }
      if (c.in(0)) store8(R(), (typename R::T *)a.dh + at + c.at(0), p[0]);
      if constexpr (GRADS) {
        if (a.want_w1) add(v, d[0]);
      }
      if (!block) continue;
      float z[1][8];  // a dh yh
#pragma unroll
      for (int e = 0; e < 8; ++e) z[0][e] = a.res_scale * y[0][e] * p[0][e];
      if constexpr (GRADS) {
        if (a.want_w2 || a.want_gate) {
          float f[1][8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[0][e] = gt * z[0][e];
          if (a.gate_mode == BN_GATE_FULL) times<E>(f, x.g, 0.0f);
          add(NV + v, f[0]);
        }
      }
      if (a.dgate && a.gate_mode == BN_GATE_FULL) {
        if (a.w_post) times<E>(z, x.w2, a.off);
        if (c.in(0)) store8(E(), (typename E::T *)a.dgate + at + c.at(0), z[0]);
      }
      if (!a.dy) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[0][e] = k[0][e] * kf * p[0][e];
      if (a.post) {  // (else y, which dgate reads, may be infinite)
#pragma unroll
        for (int e = 0; e < 8; ++e) p[0][e] = __builtin_fmaf(-c2, y[0][e], p[0][e]);
      }
      if (c.in(0)) store8(E(), (typename E::T *)a.dy + at + c.at(0), p[0]);
    }
  }
  if constexpr (GRADS) {
    float *const out = a.part + (int64_t)blockIdx.x * D;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const BnCols<W, 1> c = cols(v);
        if (!c.in(0) || !(which == 0 ? a.want_w1 : a.want_w2 ? a.want_w2 : a.want_gate)) continue;
#pragma unroll
        for (int half = 0; half < 2; ++half)
          *(f32x4 *)(out + which * (int64_t)gridDim.x * D + c.col(0) + 4 * half) = sums[2 * (which * NV + v) + half][t];
      }
  }
}

// Sums over p < np of part[which][p][c]: 16 ranges of p, each ascending, for 64 columns a
// workgroup.
template <class E>
__global__ __launch_bounds__(256) void block_norm_cols_kernel(BlockNormBwd a, int np) {
  __shared__ f32x4 red[16][16];
  const int which = blockIdx.y, D = a.D;
  if (!(which == 0 ? a.want_w1 : a.want_w2 ? a.want_w2 : a.want_gate)) return;
  const int c = threadIdx.x & 15, s = threadIdx.x >> 4, col = blockIdx.x * 64 + 4 * c;  // (D is a multiple of 8)
  const int per = (np + 15) / 16, p0 = s * per, p1 = min(np, p0 + per);
  f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
  if (col < D) {
    const float *src = a.part + ((int64_t)which * np + p0) * D + col;
#pragma unroll 16
    for (int p = p0; p < p1; ++p, src += D) x += *(const f32x4 *)src;
  }
  red[s][c] = x;
  __syncthreads();
  if (s != 0 || col >= D) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) x += red[k][c];
  if (which == 0) {
    *(f32x4 *)(a.want_w1 + col) = x;
    return;
  }
  const bool channel = a.gate_mode == BN_GATE_CHANNEL;
  f32x4 w2 = x, wg = x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (channel) w2[e] *= E::to_float(((const typename E::T *)a.gate)[col + e]);
    if (a.w_post) wg[e] *= E::to_float(((const typename E::T *)a.w_post)[col + e]) + a.off;
  }
  if (a.want_w2) *(f32x4 *)(a.want_w2 + col) = w2;
  if (a.want_gate) *(f32x4 *)(a.want_gate + col) = wg;
}

// Workgroups that sum over rows: one a CU, one vector a lane where the row allows it, as many waves as the
// registers of two sums leave room for (8192 x 2048 in bf16 49.2 us in 12 waves, 53.8 in 8; 4096 x 2048 with an fp32
// stream 34.8 in 8, 36 in 12, 39 in 16, with two vectors 41, the next row's loads ahead 34.0, but 36.8 in the
// place of 32.7 for 4096 x 3072 in bf16 from 8 bits).  Rows of 6 vectors in 12 waves, two at a time: in 8
// waves, one at a time and a quarter of the lanes idle, 42.6 for 32.7.
constexpr int BNB_PARTS = 256;
static BnShape grads_shape(int64_t D) {
  const int64_t n = (D + 511) / 512;
  if (n <= 1) return {1, 1};
  if (n <= 2) return {2, 1};
  if (n <= 3) return {3, 1};
  if (n <= 4) return {4, 1};
  if (n <= 6) return {6, 1};
  if (n <= 8) return {8, 1};
  if (n <= 12) return {12, 1};
  if (n <= 16) return {8, 2};
  return {32, 1};  // (two passes)
}

static int grads_parts(int64_t T, int64_t D, bool wide) {
  const int rows = bnb_rows(grads_shape(D).w, true, wide);
  return (int)std::min<int64_t>((T + rows - 1) / rows, BNB_PARTS);
}
// (for any types: an fp32 stream has at least as many)
int block_norm_parts(int64_t T, int64_t D) { return grads_parts(T, D, true); }

template <class E, class R, bool GRADS>
static hipError_t bwd_long(const BlockNormBwd &a, int grid, hipStream_t st) {
#define LONG(W, NV) hipLaunchKernelGGL((block_norm_bwd_long_kernel<E, R, W, NV, GRADS>), dim3(grid), dim3(64 * W), 0, st, a)
  if constexpr (E::VEC == 4) LONG(8, 4);
  else if (a.D <= 12288) LONG(12, 2);
  else LONG(16, 2);
#undef LONG
  return hipGetLastError();
}

template <class E, class R>
static hipError_t bwd_grads(const BlockNormBwd &a, hipStream_t st) {
  const BnShape s = grads_shape(a.D);
  constexpr bool wide = R::VEC == 4;
  const int np = grads_parts(a.T, a.D, wide);
  hipError_t e = hipSuccess;
#define BWD(W, NV) hipLaunchKernelGGL((block_norm_bwd_kernel<E, R, W, NV, true, false>), dim3(np), dim3(bnb_threads(W, true, wide)), 0, st, a)
  switch (s.w * 8 + s.nv) {
    case 1 * 8 + 1: BWD(1, 1); break;
    case 2 * 8 + 1: BWD(2, 1); break;
    case 3 * 8 + 1: BWD(3, 1); break;
    case 4 * 8 + 1: BWD(4, 1); break;
    case 6 * 8 + 1: BWD(6, 1); break;
    case 8 * 8 + 1: BWD(8, 1); break;
    case 12 * 8 + 1: BWD(12, 1); break;
    case 8 * 8 + 2: BWD(8, 2); break;
    default: e = bwd_long<E, R, true>(a, np, st); break;
  }
#undef BWD
  if (e != hipSuccess || (e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL((block_norm_cols_kernel<E>), dim3((a.D + 63) / 64, 2), dim3(256), 0, st, a, np);
  return hipGetLastError();
}

// Waves a row and vectors a lane without sums over rows.  A stream of fp32 leaves registers for one vector a
// lane (8192 x 2048 57.5 us, two 64.5; 4096 x 2048 all fp32 40.1, 53.3), one of bf16 for two (4096 x 3072 from
// 8 bits 25.1, one 34.2) up to 4096 columns; beyond them more waves are faster (2048 x 5632 from
// 8 bits 32.6 in 12 waves, 35.8 in 6; 2048 x 8192 with an fp32 stream 70 in 16, 76 in 8).
static BnShape rows_shape(int64_t T, int64_t D, bool wide) {
  const int64_t n = (D + 511) / 512;
  if (T * n <= 1024 && n <= 8) return bn_shape(T, D);
  if (n <= 1) return {1, 1};
  if (n <= 8 && !wide) return bn_shape(T, D);
  if (n <= 4) return {(int)n, 1};
  if (n <= 6) return {6, 1};
  if (n <= 8) return {8, 1};
  if (n <= 12) return {12, 1};
  if (n <= 16) return {16, 1};
  return {12, 2};
}

template <class E, class R>
static hipError_t bwd_rows(const BlockNormBwd &a, hipStream_t st) {
  if (a.want_w1 || a.want_w2 || a.want_gate) return bwd_grads<E, R>(a, st);
  constexpr bool wide = R::VEC == 4;
  if (a.D > (wide ? 8192 : 12288)) return bwd_long<E, R, false>(a, (int)std::min<int64_t>(a.T, 1 << 16), st);
  const BnShape s = rows_shape(a.T, a.D, wide);
  const dim3 grid((unsigned)std::min(s.w == 1 ? (a.T + 3) / 4 : a.T, BN_GRID_ROWS));
  // What is large and read once goes past the caches, which what is written then has: 4096 x 3072 from 8 bits 25.2 us
  // for 27.6, 4096 x 2048 22.2 for 22.9.  (With sums over rows it gains nothing, 35.5 for 35.3.)
  const bool once = a.T * (int64_t)a.D >= (int64_t)1 << 23;
#define BWD(W, NV)                                                                                                     \
  case W * 8 + NV:                                                                                                     \
    if (once)                                                                                                          \
      hipLaunchKernelGGL((block_norm_bwd_kernel<E, R, W, NV, false, true>), grid, dim3(bnb_threads(W, false, wide)), 0, st, a); \
    else                                                                                                               \
      hipLaunchKernelGGL((block_norm_bwd_kernel<E, R, W, NV, false, false>), grid, dim3(bnb_threads(W, false, wide)), 0, st, a); \
    break;
  if constexpr (wide) {
    switch (s.w * 8 + s.nv) {
      BWD(1, 1) BWD(2, 1) BWD(3, 1) BWD(4, 1) BWD(6, 1) BWD(8, 1) BWD(12, 1) BWD(16, 1)
      default: return hipErrorInvalidValue;
    }
  } else {
    switch (s.w * 8 + s.nv) {
      BWD(1, 1) BWD(4, 1) BWD(8, 1) BWD(12, 1) BWD(16, 1) BWD(1, 2) BWD(2, 2) BWD(3, 2) BWD(4, 2) BWD(12, 2)
      default: return hipErrorInvalidValue;
    }
  }
#undef BWD
  return hipGetLastError();
}

hipError_t launch_block_norm_bwd(const BlockNormBwd &a, Dtype d, Dtype res, hipStream_t st) {
  if (d == DT_F32) return bwd_rows<F32, F32>(a, st);
  return res == DT_F32 ? bwd_rows<BF16, F32>(a, st) : bwd_rows<BF16, BF16>(a, st);
}

}  // namespace lora
