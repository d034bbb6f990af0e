// tokenloss.hip -- log-probabilities of given tokens under rows of logits, and
// the policy and preference losses over them with their gradients with
// respect to the logits.
//   m_t = max_j z_tj,  l_t = log sum_j exp(z_tj - m_t),
//   logp_t = (z_t[y_t] - m_t) - l_t
//   dz_tj = c_t ([j = y_t] - exp((z_tj - m_t) - l_t)),   c_t = w_t dL_t/dlogp_t
// m and l are kept apart: a row whose logits are all the type's lowest value
// has the finite m of that size, beside which l would be rounded away.
// Differences are taken before the scaling to base 2 for the same reason.
// Rows of weight 0 are not read; their logp is 0 and their gradient a row of zeros.
#include "kernels.hpp"
#include "launch.hpp"

namespace lora {

constexpr float kLog2e = 1.44269504088896340736f;

// Running maximum and sum of exp(z - m).  A lane that has seen nothing (or only
// -inf) has m = -inf and s = 0 (exponents are taken from 0 then).
struct Stat {
  float m, s;
};
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ float exp_diff(float z, float m) { return __builtin_amdgcn_exp2f((z - m) * kLog2e); }
__device__ __forceinline__ Stat stat_join(Stat a, Stat b) {
  const float m = fmaxf(a.m, b.m), r = finite_max(m);
  return {m, a.s * exp_diff(a.m, r) + b.s * exp_diff(b.m, r)};
}
template <int N>
__device__ __forceinline__ void stat_add(Stat &a, const float *f) {
  float v = f[0];
#pragma unroll
  for (int e = 1; e < N; ++e) v = fmaxf(v, f[e]);
  const float m = fmaxf(a.m, v), r = finite_max(m);
  float s = a.s * exp_diff(a.m, r);
#pragma unroll
  for (int e = 0; e < N; ++e) s += exp_diff(f[e], r);
  a = {m, s};
}

template <int NT>
__device__ __forceinline__ Stat block_stat(Stat a, Stat *red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) a = stat_join(a, Stat{__shfl_xor(a.m, off), __shfl_xor(a.s, off)});
  if (NT == 64) return a;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
  __syncthreads();
  a = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) a = stat_join(a, red[w]);
  return a;
}

// Vector i of a row of V logits, -inf past its end (a row's storage is whole vectors).
template <typename E>
__device__ __forceinline__ void load_logits(const u32x4 *row, int i, int V, float *f) {
  unpack_vec(E(), row[i], f);
  if ((i + 1) * E::VEC > V) {
#pragma unroll
    for (int e = 0; e < E::VEC; ++e)
      if (i * E::VEC + e >= V) f[e] = -INFINITY;
  }
}

constexpr int TL_NT = 256;

// max and log of the sum of exponentials of a row, for the whole workgroup.
template <typename E>
__device__ __forceinline__ Stat row_stat(const u32x4 *row, int V, Stat *red) {
  Stat a{-INFINITY, 0.0f};
  const int nv = (V + E::VEC - 1) / E::VEC;
  for (int i = threadIdx.x; i < nv; i += TL_NT) {
    float f[E::VEC];
    load_logits<E>(row, i, V, f);
    stat_add<E::VEC>(a, f);
  }
  a = block_stat<TL_NT>(a, red);
  return {a.m, logf(a.s)};
}

template <typename E>
__device__ __forceinline__ float target_logp(const TokenLoss &a, int64_t t, Stat st) {
  const int y = a.y[t];
  if (y < 0 || y >= a.V) return NAN;
  return (E::to_float(((const typename E::T *)a.z)[t * a.ld + y]) - st.m) - st.s;
}

// Row t of dz from its statistics and c.
template <typename E>
__device__ __forceinline__ void write_dz(const TokenLoss &a, int64_t t, Stat st, float c) {
  const int nv = (int)(a.ld / E::VEC);
  const u32x4 *row = (const u32x4 *)((const typename E::T *)a.z + t * a.ld);
  u32x4 *out = (u32x4 *)((typename E::T *)a.dz + t * a.ld);
  if (c == 0.0f) {
    for (int i = threadIdx.x; i < nv; i += TL_NT) out[i] = zero16();
    return;
  }
  const int y = a.y[t];
  const float l2 = st.s * kLog2e;
  for (int i = threadIdx.x; i < nv; i += TL_NT) {
    u32x4 x = zero16();
    if (i * E::VEC < a.V) {
      float f[E::VEC];
      load_logits<E>(row, i, a.V, f);
#pragma unroll
      for (int e = 0; e < E::VEC; ++e) {
        const float p = __builtin_amdgcn_exp2f((f[e] - st.m) * kLog2e - l2);
        f[e] = i * E::VEC + e >= a.V ? 0.0f : -c * p;
        if (i * E::VEC + e == y) f[e] += c;
      }
      x = pack_vec(E(), f);
    }
    out[i] = x;
  }
}

// logp, and for a loss that comes later the row's statistics and a zero c.
template <typename E>
__global__ __launch_bounds__(TL_NT) void token_logp_kernel(TokenLoss a) {
  __shared__ Stat red[TL_NT / 64];
  const int64_t t = blockIdx.x;
  Stat st{0.0f, 0.0f};
  const bool live = !a.w || a.w[t] != 0.0f;
  if (live) st = row_stat<E>((const u32x4 *)((const typename E::T *)a.z + t * a.ld), a.V, red);
  if (threadIdx.x) return;
  a.logp[t] = live ? target_logp<E>(a, t, st) : 0.0f;
  if (a.stat) {
    a.stat[2 * t] = st.m;
    a.stat[2 * t + 1] = st.s;
    a.coef[t] = 0.0f;
  }
}

// The policy loss of a position and its derivative with respect to logp.
__device__ __forceinline__ void policy_terms(const PolicyArgs &p, int64_t t, float logp, float *loss, float *grad) {
  const float adv = p.adv[t], ratio = expf(logp - p.old_logp[t]);
  // (an unordered comparison takes the bound's side only when the bound is less: NaN stays NaN)
  const float held = fminf(fmaxf(ratio, p.lo), p.hi) * adv, free = ratio * adv;
  const bool clipped = held < free;
  float l = clipped ? -held : -free, g = clipped ? 0.0f : -free;
  if (p.ref) {
    const float d = p.ref[t] - logp, x = expm1f(d);
    l += p.kl * (x - d);
    g -= p.kl * x;
  }
  *loss = l;
  *grad = g;
}

template <typename E>
__global__ __launch_bounds__(TL_NT) void policy_kernel(TokenLoss a, PolicyArgs p) {
  __shared__ Stat red[TL_NT / 64];
  const int64_t t = blockIdx.x;
  const float w = a.w ? a.w[t] : 1.0f;
  Stat st{0.0f, 0.0f};
  float c = 0.0f;
  if (w != 0.0f) {
    st = row_stat<E>((const u32x4 *)((const typename E::T *)a.z + t * a.ld), a.V, red);
    const float logp = target_logp<E>(a, t, st);
    float l, g;
    policy_terms(p, t, logp, &l, &g);
    c = w * g;
    if (threadIdx.x == 0) {
      a.logp[t] = logp;
      a.rows[t] = w * l;
    }
  } else if (threadIdx.x == 0) {
    a.logp[t] = 0.0f;
    a.rows[t] = 0.0f;
  }
  if (a.dz) {
    __syncthreads();  // dz may be z: every thread has the target's logit before its row changes
    write_dz<E>(a, t, st, c);
  }
}

template <typename E>
__global__ __launch_bounds__(TL_NT) void token_dz_kernel(TokenLoss a) {
  const int64_t t = blockIdx.x;
  write_dz<E>(a, t, Stat{a.stat[2 * t], a.stat[2 * t + 1]}, a.coef[t]);
}

// Sum over a workgroup of NT threads in a fixed order.
template <int NT>
__device__ __forceinline__ double block_sum(double x, double *red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) x += red[w];
  return x;
}

constexpr int LS_NT = 1024;
// loss = scale * sum of rows[0 .. n), by one workgroup.
__global__ __launch_bounds__(LS_NT) void loss_sum_kernel(const float *rows, int n, double scale, float *loss) {
  __shared__ double red[LS_NT / 64];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += LS_NT) s += rows[i];
  s = block_sum<LS_NT>(s, red);
  if (threadIdx.x == 0) loss[0] = (float)(s * scale);
}

// softplus(x) = log(1 + exp x)
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.0f) + log1pf(expf(-fabsf(x))); }

// One workgroup a pair: margin, loss and the rows' c.
__global__ __launch_bounds__(TL_NT) void pair_kernel(TokenLoss a, PairArgs p) {
  __shared__ double red[TL_NT / 64];
  const int i = blockIdx.x;
  const int b0 = min(max(p.seq[2 * i], 0), a.T), b1 = min(max(p.seq[2 * i + 1], b0), a.T), b2 = min(max(p.seq[2 * i + 2], b1), a.T);
  double d = 0.0;
  for (int t = b0 + threadIdx.x; t < b2; t += TL_NT) {
    const float w = a.w ? a.w[t] : 1.0f;
    if (w == 0.0f) continue;
    const double x = (double)w * ((double)a.logp[t] - (p.ref ? (double)p.ref[t] : 0.0));
    d += t < b1 ? x : -x;
  }
  const float margin = p.beta * (float)block_sum<TL_NT>(d, red);
  const float s = p.smooth, up = 1.0f / (1.0f + expf(-margin)), down = 1.0f / (1.0f + expf(margin));
  const float g = p.beta / p.pairs * (s * up - (1.0f - s) * down);
  for (int t = b0 + threadIdx.x; t < b2; t += TL_NT) {
    const float w = a.w ? a.w[t] : 1.0f;
    a.coef[t] = w == 0.0f ? 0.0f : w * (t < b1 ? g : -g);
  }
  if (threadIdx.x == 0) {
    p.margins[i] = margin;
    float l = (1.0f - s) * softplus(-margin);
    if (s != 0.0f) l += s * softplus(margin);
    a.rows[i] = l;
  }
}

hipError_t launch_token_logp(const TokenLoss &a, Dtype d, hipStream_t st) {
  if (d == DT_BF16) hipLaunchKernelGGL(token_logp_kernel<BF16>, dim3(a.T), dim3(TL_NT), 0, st, a);
  else hipLaunchKernelGGL(token_logp_kernel<F32>, dim3(a.T), dim3(TL_NT), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_policy_loss(const TokenLoss &a, const PolicyArgs &p, Dtype d, hipStream_t st) {
  if (d == DT_BF16) hipLaunchKernelGGL(policy_kernel<BF16>, dim3(a.T), dim3(TL_NT), 0, st, a, p);
  else hipLaunchKernelGGL(policy_kernel<F32>, dim3(a.T), dim3(TL_NT), 0, st, a, p);
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(LS_NT), 0, st, a.rows, a.T, 1.0, a.loss);
  return hipGetLastError();
}

hipError_t launch_preference_loss(const TokenLoss &a, const PairArgs &p, Dtype d, hipStream_t st) {
  hipError_t e = launch_token_logp(a, d, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pair_kernel, dim3(p.pairs), dim3(TL_NT), 0, st, a, p);
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(LS_NT), 0, st, a.rows, p.pairs, 1.0 / p.pairs, a.loss);
  if (a.dz) {
    if (d == DT_BF16) hipLaunchKernelGGL(token_dz_kernel<BF16>, dim3(a.T), dim3(TL_NT), 0, st, a);
    else hipLaunchKernelGGL(token_dz_kernel<F32>, dim3(a.T), dim3(TL_NT), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace lora
