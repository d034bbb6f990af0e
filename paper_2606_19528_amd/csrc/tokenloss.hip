// tokenloss.hip -- log-probabilities of given tokens under rows of logits, and
// the policy and preference losses over them with their gradients with
// respect to the logits.
//   m_t = max_j z_tj,  s_t = sum_j exp(z_tj - m_t),
//   logp_t = (z_t[y_t] - m_t) - log s_t
//   dz_tj = c_t [j = y_t] - (c_t / s_t) exp(z_tj - m_t),   c_t = w_t dL_t/dlogp_t
// m and s are kept apart: a row whose logits are all the type's lowest value
// has the finite m of that size, beside which log s would be rounded away.
// Differences are taken before the scaling to base 2 for the same reason.
// logp is held in 64 bits until it is rounded for the output: in 32 bits the rounding of
// log s and logp would be most of the error of a margin, a difference of sums of logp.
// Rows of weight 0 are not read; their logp is 0 and their gradient a row of zeros.
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "launch.hpp"
#include "meet_flags.hpp"

namespace lora {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLog2eRest = 1.925963033500011e-8f;  // log2 e - kLog2e

// Running maximum and sum of exp(z - m).  A lane that has seen nothing (or only
// -inf) has m = -inf and s = 0 (exponents are taken from 0 then).
struct Stat {
  float m, s;
};
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }
// exp(z - m).  Scaled by kLog2e alone every term would be high by 1.3e-8 (m - z) of itself, and
// log s by that times the mean of m - z: about 6e-8 in every row of a decoder's logits, which
// a margin, a difference of sums over rows, adds up instead of averaging.
__device__ __forceinline__ float exp_diff(float z, float m) {
  const float d = z - m;
  return __builtin_amdgcn_exp2f(fmaf(d, kLog2e, d * kLog2eRest));
}
// The same where it is one element's factor (dz): the offset is below the rounding of the product.
__device__ __forceinline__ float exp_diff_fast(float z, float m) { return __builtin_amdgcn_exp2f((z - m) * kLog2e); }
__device__ __forceinline__ Stat stat_join(Stat a, Stat b) {
  const float m = fmaxf(a.m, b.m), r = finite_max(m);
  return {m, a.s * exp_diff(a.m, r) + b.s * exp_diff(b.m, r)};
}
// U statistics, each joined over groups of `width` lanes (a power of two).  First to the common
// maximum, then plain sums: both give every lane the same bits, since a + b = b + a.  (A
// multiply-add of the lane's own product and its partner's rounded one rounds differently in the
// two lanes, and lanes that take different sides of a clip leave a row of dz partly zero.)
template <int U>
__device__ __forceinline__ void group_stats(Stat (&x)[U], int width) {
#pragma clang fp contract(off)
  float m[U];
#pragma unroll
  for (int u = 0; u < U; ++u) m[u] = x[u].m;
  for (int off = width >> 1; off >= 1; off >>= 1)
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = fmaxf(m[u], __shfl_xor(m[u], off));
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = {m[u], x[u].s * exp_diff(x[u].m, finite_max(m[u]))};
  for (int off = width >> 1; off >= 1; off >>= 1)
#pragma unroll
    for (int u = 0; u < U; ++u) x[u].s += __shfl_xor(x[u].s, off);
}
__device__ __forceinline__ Stat wave_stat(Stat a) {
  Stat x[1] = {a};
  group_stats<1>(x, 64);
  return x[0];
}
template <int N>
__device__ __forceinline__ float max_of(const float *f) {
  float v = f[0];
#pragma unroll
  for (int e = 1; e < N; ++e) v = fmaxf(v, f[e]);
  return v;
}
template <int N>
__device__ __forceinline__ void stat_add(Stat &a, const float *f) {
  const float m = fmaxf(a.m, max_of<N>(f)), r = finite_max(m);
  float s = a.s * exp_diff(a.m, r);
#pragma unroll
  for (int e = 0; e < N; ++e) s += exp_diff(f[e], r);
  a = {m, s};
}
// Joined over a workgroup of NT threads, in one order.
template <int NT>
__device__ __forceinline__ Stat block_stat(Stat a, Stat *red) {
  a = wave_stat(a);
  if (NT == 64) return a;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
  __syncthreads();
  a = red[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) a = stat_join(a, red[w]);
  return a;
}

// Vector i of a row of V elements with those past the row's end replaced by the
// bits `fill` (a row's storage is whole vectors).
__device__ __forceinline__ u32x4 cut_row(BF16, u32x4 x, int i, int V, uint32_t fill) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    if (i * 8 + 2 * d + 1 >= V) x[d] = (x[d] & 0xffffu) | (fill << 16);
    if (i * 8 + 2 * d >= V) x[d] = fill | (fill << 16);
  }
  return x;
}
__device__ __forceinline__ u32x4 cut_row(F32, u32x4 x, int i, int V, uint32_t fill) {
#pragma unroll
  for (int d = 0; d < 4; ++d)
    if (i * 4 + d >= V) x[d] = fill;
  return x;
}
__device__ __forceinline__ uint32_t neg_inf_bits(BF16) { return 0xff80u; }
__device__ __forceinline__ uint32_t neg_inf_bits(F32) { return 0xff800000u; }
// A vector of logits into the statistics.
template <typename E>
__device__ __forceinline__ void stat_vec(Stat &st, u32x4 x) {
  float f[E::VEC];
  unpack_vec(E(), x, f);
  stat_add<E::VEC>(st, f);
}
__device__ __forceinline__ u32x4 pack_pairs(BF16, const float *f) {
  return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}
__device__ __forceinline__ u32x4 pack_pairs(F32, const float *f) { return pack_vec(F32(), f); }
// Vector i of dz (k = -c / s), elements past the row's end included.
template <typename E>
__device__ __forceinline__ u32x4 dz_vec(u32x4 x, int i, float m, float k, float c, int y) {
  float f[E::VEC];
  unpack_vec(E(), x, f);
#pragma unroll
  for (int e = 0; e < E::VEC; ++e) f[e] = k * exp_diff_fast(f[e], m);
  const int ye = y - i * E::VEC;
  if ((unsigned)ye < (unsigned)E::VEC) {
#pragma unroll
    for (int e = 0; e < E::VEC; ++e)
      if (e == ye) f[e] += c;
  }
  return pack_pairs(E(), f);
}

template <typename E>
__device__ __forceinline__ const u32x4 *row_ptr(const TokenLoss &a, int64_t t) {
  return (const u32x4 *)((const typename E::T *)a.z + t * a.ld);
}
template <typename E>
__device__ __forceinline__ u32x4 *dz_ptr(const TokenLoss &a, int64_t t) {
  return (u32x4 *)((typename E::T *)a.dz + t * a.ld);
}
__device__ __forceinline__ float weight(const TokenLoss &a, int64_t t) { return a.w ? a.w[t] : 1.0f; }

// The target's logit of row t; NaN for a target outside the vocabulary.
template <typename E>
__device__ __forceinline__ float target_logit(const TokenLoss &a, int64_t t) {
  const int y = a.y[t];
  return y >= 0 && y < a.V ? E::to_float(((const typename E::T *)a.z)[t * a.ld + y]) : NAN;
}
// log s to fp32's relative precision of s itself: the hardware's base-2 logarithm,
// corrected by what s 2^-l2 leaves of 1 (its square is below 2^-40).
__device__ __forceinline__ double log_sum(float s) {
  const float l2 = __builtin_amdgcn_logf(s);
  const float e = fmaf(s, __builtin_amdgcn_exp2f(-l2), -1.0f);
  return (double)l2 * 0.6931471805599453094 + (double)e;
}
__device__ __forceinline__ double logp_of(float zy, Stat st) { return ((double)zy - (double)st.m) - log_sum(st.s); }

// The policy loss of a position and its derivative with respect to logp.
__device__ __forceinline__ void policy_terms(const PolicyArgs &p, int64_t t, double logp, float *loss, float *grad) {
  const float adv = p.adv[t], ratio = expf((float)(logp - (double)p.old_logp[t]));
  // (an unordered comparison does not clip: NaN stays NaN)
  const float held = fminf(fmaxf(ratio, p.lo), p.hi) * adv, free = ratio * adv;
  const bool clipped = held < free;
  float l = clipped ? -held : -free, g = clipped ? 0.0f : -free;
  if (p.ref) {
    const float d = (float)((double)p.ref[t] - logp), x = expm1f(d);
    l += p.kl * (x - d);
    g -= p.kl * x;
  }
  *loss = l;
  *grad = g;
}

// ---- statistics of rows, or of parts of rows -------------------------------------
// Bound by reading the logits: 4096 x 151936 bf16, three quarters of them live, 167 us (933 MB,
// 5.6 TB/s; 166 with one operation a logit less, log2 e in one term).  One pass: each thread keeps a running maximum and a sum relative to it,
// joined over lanes, waves and parts.
constexpr int TL_NT = 256;

// Part p of row t, vectors [p, p + 1) part_vecs, for the whole workgroup.
template <typename E>
__device__ __forceinline__ Stat part_stat(const TokenLoss &a, int64_t t, int p, Stat *red) {
  const u32x4 *row = row_ptr<E>(a, t);
  const int nv = (a.V + E::VEC - 1) / E::VEC, end = min(nv, (p + 1) * a.part_vecs);
  Stat st{-INFINITY, 0.0f};
  for (int i = p * a.part_vecs + threadIdx.x; i < end; i += TL_NT) {
    u32x4 x = row[i];
    if ((i + 1) * E::VEC > a.V) x = cut_row(E(), x, i, a.V, neg_inf_bits(E()));
    stat_vec<E>(st, x);
  }
  return block_stat<TL_NT>(st, red);
}

// stat: for the launches that follow; null: whole rows, logp.
template <typename E>
__global__ __launch_bounds__(TL_NT) void token_stat_kernel(TokenLoss a, Stat *stat) {
  __shared__ Stat red[TL_NT / 64];
  const int64_t t = blockIdx.x / a.parts;
  const int p = blockIdx.x % a.parts;
  if (a.coef && p == 0 && threadIdx.x == 0) {
    a.coef[t] = 0.0f;
    if (t == 0) a.coef[a.T] = 0.0f;  // (pair_kernel: offsets that are not ascending)
  }
  if (weight(a, t) == 0.0f) {
    if (!stat && threadIdx.x == 0) a.logp[t] = 0.0f;
    return;
  }
  const Stat st = part_stat<E>(a, t, p, red);
  if (threadIdx.x) return;
  if (stat) stat[blockIdx.x] = st;
  else a.logp[t] = (float)logp_of(target_logit<E>(a, t), st);
  // (a later launch may put dz in the logits' place, one part before another)
  if (stat && p == 0) a.ztgt[t] = target_logit<E>(a, t);
}

// A row's statistics from those of its parts (at most 64): in every lane of a
// wave, the same bits, or by one thread.
__device__ __forceinline__ Stat joined_stat(const TokenLoss &a, const Stat *stat, int64_t t) {
  const int lane = threadIdx.x & 63;
  return wave_stat(lane < a.parts ? stat[t * a.parts + lane] : Stat{-INFINITY, 0.0f});
}
__device__ __forceinline__ Stat thread_stat(const TokenLoss &a, const Stat *stat, int64_t t) {
  constexpr int U = 8;  // loads in flight
  Stat st{-INFINITY, 0.0f};
  for (int p = 0; p < a.parts; p += U) {
    Stat x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = stat[t * a.parts + min(p + u, a.parts - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p + u < a.parts) st = stat_join(st, x[u]);
  }
  return st;
}

// token_logp of few rows in one launch: the parts of a row meet (meet.hpp), and the
// one that comes last joins them.  Statistics and flags are written and read at
// device scope, by the first wave.
template <typename E>
__global__ __launch_bounds__(TL_NT) void logp_parts_kernel(TokenLoss a) {
  __shared__ Stat red[TL_NT / 64];
  const int64_t t = blockIdx.x / a.parts;
  const int p = blockIdx.x % a.parts, lane = threadIdx.x & 63;
  if (weight(a, t) == 0.0f) {
    if (p == 0 && threadIdx.x == 0) a.logp[t] = 0.0f;
    return;
  }
  const Stat st = part_stat<E>(a, t, p, red);
  if (threadIdx.x >= 64) return;
  uint64_t *slot = (uint64_t *)a.stat + t * a.parts;
  if (lane == 0) __hip_atomic_store(slot + p, __builtin_bit_cast(uint64_t, st), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  MeetFlags flags{a.sync + t * a.parts, lane};
  flags.settle();  // the part is in memory before its flag rises
  if (!meet_arrive(flags, p, a.parts, a.gen)) return;
  Stat all{-INFINITY, 0.0f};
  if (lane < a.parts)
    all = __builtin_bit_cast(Stat, __hip_atomic_load(slot + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  all = wave_stat(all);
  const float logp = (float)logp_of(target_logit<E>(a, t), all);
  if (meet_lower(flags, a.parts) == a.gen && lane == 0) a.logp[t] = logp;
}

// ---- sums over positions -----------------------------------------------------------
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
// loss = scale * sum of rows[0 .. n), by one workgroup.
template <int NT>
__device__ __forceinline__ void sum_rows(const float *rows, int64_t n, double scale, float *loss, double *red) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += NT) s += rows[i];
  s = block_sum<NT>(s, red);
  if (threadIdx.x == 0) loss[0] = (float)(s * scale);
}

constexpr int LS_NT = 1024;
__global__ __launch_bounds__(LS_NT) void loss_sum_kernel(const float *rows, int n, double scale, float *loss) {
  __shared__ double red[LS_NT / 64];
  sum_rows<LS_NT>(rows, n, scale, loss, red);
}

// ---- dz in a launch after the statistics ---------------------------------------------
// Part p of row t of dz from its maximum m, sum s and c, by a workgroup.  NTS:
// stores that pass the last-level cache by.
template <bool NTS>
__device__ __forceinline__ void put_dz(u32x4 d, u32x4 *out) {
  if (NTS) __builtin_nontemporal_store(d, out);
  else *out = d;
}
template <typename E, bool NTS>
__device__ __forceinline__ void write_dz(const TokenLoss &a, int64_t t, int p, Stat st, float c, int y) {
  const int nv = (int)(a.ld / E::VEC), nz = (a.V + E::VEC - 1) / E::VEC;
  const int end = p + 1 == a.parts ? nv : min(nv, (p + 1) * a.part_vecs);
  const u32x4 *row = row_ptr<E>(a, t);
  u32x4 *out = dz_ptr<E>(a, t);
  int i = p * a.part_vecs + threadIdx.x;
  if (c != 0.0f) {
    const float k = -c / st.s;
    for (; i < end && i < nz; i += TL_NT) {
      u32x4 d = dz_vec<E>(row[i], i, st.m, k, c, y);
      if ((i + 1) * E::VEC > a.V) d = cut_row(E(), d, i, a.V, 0u);
      put_dz<NTS>(d, out + i);
    }
  }
  for (; i < end; i += TL_NT) put_dz<NTS>(zero16(), out + i);
}

// From this many rows on, rows in registers; fewer in parts.  128256 columns, us a call in registers /
// in parts: bf16 128 rows 32 / 20, 193 35 / 29, 256 38 / 37, 300 64 / 49, 512 66 / 72, 513 84 /
// 76; fp32 128 38 / 38, 193 54 / 56, 256 62 / 74, 300 101 / 87, 512 128 / 147.  A row takes a whole
// CU's registers, so rows come in rounds of 256, which this rule does not follow.
constexpr int POLICY_ROWS = 192;
static_assert(POLICY_ROWS <= TL_NT, "a thread a row");

// Bound by launches and latency: 97 x 8192 fp32 3.9 + 4.7 us on the GPU, 11.7 a call.
// Policy loss of few rows, after token_stat_kernel: each workgroup writes one
// part of a row of dz; ahead of them the first one sums the loss, and LOSS_WGS - 1 end at once:
// a part is read again on the XCD, one of 8 in turn, whose cache has it from the statistics (60 x
// 151936 fp32 20.3 us a call, 21.9 with one workgroup ahead).
constexpr int LOSS_WGS = 8;
template <typename E>
__global__ __launch_bounds__(TL_NT) void policy_parts_kernel(TokenLoss a, PolicyArgs p, const Stat *stat) {
  __shared__ double red[TL_NT / 64];
  __shared__ Stat rows[POLICY_ROWS];
  if (blockIdx.x == 0) {
    // Statistics of the rows, `width` lanes each, joined as joined_stat does (empty lanes change
    // no bits), so that the loss takes the same side of the clip as dz; then a thread a row.
    constexpr int WAVES = TL_NT / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int width = a.parts > 1 ? 1 << (32 - __clz(a.parts - 1)) : 1, per = 64 / width, part = lane % width;
    int t0 = wave * per + lane / width;
    auto join = [&](auto n) {  // n rows of each group of lanes at once
      constexpr int U = decltype(n)::value;
      Stat x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = stat[min(t0 + u * WAVES * per, a.T - 1) * a.parts + min(part, a.parts - 1)];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (part >= a.parts) x[u] = Stat{-INFINITY, 0.0f};
      group_stats<U>(x, width);
#pragma unroll
      for (int u = 0; u < U; ++u, t0 += WAVES * per)
        if (part == 0 && t0 < a.T) rows[t0] = x[u];
    };
    int left = (a.T + WAVES * per - 1) / (WAVES * per);
    for (; left > 2; left -= 8) join(std::integral_constant<int, 8>());
    if (left > 0) join(std::integral_constant<int, 2>());
    __syncthreads();
    double sum = 0.0;
    const int t = threadIdx.x;
    if (t < a.T) {
      const float w = weight(a, t);
      double logp = 0.0;
      if (w != 0.0f) {
        float l, g;
        logp = logp_of(a.ztgt[t], rows[t]);
        policy_terms(p, t, logp, &l, &g);
        sum = w * l;
      }
      a.logp[t] = (float)logp;
    }
    sum = block_sum<TL_NT>(sum, red);
    if (threadIdx.x == 0) a.loss[0] = (float)sum;
    return;
  }
  if (blockIdx.x < LOSS_WGS) return;
  const unsigned b = blockIdx.x - LOSS_WGS;
  const int64_t t = b / a.parts;
  const float w = weight(a, t);
  Stat st{0.0f, 1.0f};
  float c = 0.0f;
  int y = -1;
  if (w != 0.0f) {
    float l, g;
    st = joined_stat(a, stat, t);
    policy_terms(p, t, logp_of(a.ztgt[t], st), &l, &g);
    c = w * g;
    y = a.y[t];
  }
  write_dz<E, false>(a, t, b % a.parts, st, c, y);
}

// softplus(x) = log(1 + exp x)
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.0f) + log1pf(expf(-fabsf(x))); }

// One workgroup a pair, a thread a row: logp and statistics of its rows, margin,
// loss and the rows' c.  The first and the last pair take the rows outside all of
// them along (their c is 0: token_stat_kernel).
constexpr int PR_NT = 512;
__global__ __launch_bounds__(PR_NT) void pair_kernel(TokenLoss a, PairArgs p, const Stat *stat, Stat *rowstat) {
  __shared__ double red[PR_NT / 64];
  const int i = blockIdx.x;
  const int s0 = p.seq[2 * i], s1 = p.seq[2 * i + 1], s2 = p.seq[2 * i + 2];
  const int b0 = min(max(s0, 0), a.T), b1 = min(max(s1, b0), a.T), b2 = min(max(s2, b1), a.T);
  const int64_t first = i == 0 ? 0 : b0, last = i == p.pairs - 1 ? a.T : b2;
  double d = 0.0;
  for (int64_t t = first + threadIdx.x; t < last; t += PR_NT) {
    const float w = weight(a, t);
    double logp = 0.0;
    if (w != 0.0f) {
      const Stat st = thread_stat(a, stat, t);
      logp = logp_of(a.ztgt[t], st);
      rowstat[t] = st;
      if (t >= b0 && t < b2) {
        const double x = (double)w * (logp - (p.ref ? (double)p.ref[t] : 0.0));
        d += t < b1 ? x : -x;
      }
    }
    a.logp[t] = (float)logp;
  }
  const double margin = (double)p.beta * block_sum<PR_NT>(d, red);
  const float mg = (float)margin, s = p.smooth, up = 1.0f / (1.0f + expf(-mg)), down = 1.0f / (1.0f + expf(mg));
  const float g = p.beta / p.pairs * (s * up - (1.0f - s) * down);
  for (int64_t t = b0 + threadIdx.x; t < b2; t += PR_NT) {
    const float w = weight(a, t);
    if (w != 0.0f) a.coef[t] = w * (t < b1 ? g : -g);
  }
  if (threadIdx.x == 0) {
    float l = (1.0f - s) * softplus(-mg);
    if (s != 0.0f) l += s * softplus(mg);
    // Offsets that fall at this pair: another one may hold the same rows, and which of the
    // two leaves their c is left to chance.  The loss and every c are NaN then.
    const bool falls = s1 < s0 || s2 < s1;
    if (falls) a.coef[a.T] = NAN;
    p.margins[i] = falls ? NAN : mg;
    a.rows[i] = falls ? NAN : l;
  }
}

// Bound by memory: of 2048 x 151936 bf16 in four pairs 373 MB are read and 622 written in 185 us
// (5.4 TB/s) after 60 us of statistics and 6 of pair_kernel.
// dz, and by the last workgroup the loss.  The rows go backwards: the last ones
// that token_stat_kernel read may still be in the last-level cache.
template <typename E, bool NTS>
__global__ __launch_bounds__(TL_NT) void pair_dz_kernel(TokenLoss a, const Stat *rowstat, int pairs) {
  __shared__ double red[TL_NT / 64];
  if (blockIdx.x == gridDim.x - 1) {
    sum_rows<TL_NT>(a.rows, pairs, 1.0 / pairs, a.loss, red);
    return;
  }
  const unsigned b = gridDim.x - 2 - blockIdx.x;
  const int64_t t = b / a.parts;
  const float c = a.coef[t] + a.coef[a.T];
  write_dz<E, NTS>(a, t, b % a.parts, c != 0.0f ? rowstat[t] : Stat{0.0f, 1.0f}, c, a.y[t]);
}

// ---- policy loss of many rows: a row stays in registers -------------------------------
// A workgroup of NT threads holds a row of up to NT NV vectors, so the logits
// are read once.  A row's vectors are replaced by the next row's as they are
// turned into dz, which keeps loads and stores in flight while the exponentials
// are computed.  Rows are addressed as buffers of their own length: what a
// thread loads past the end is 0, what it stores there is dropped, and the
// vectors need one address register.  What a longer row has beyond is read
// twice; with one row a CU on the way, the second read comes from the last-level cache.
// Bound by memory: 4096 x 128256 bf16, three quarters live, 365 - 380 us (1.84 GB, 4.8 - 5.0 TB/s, a
// copy's rate), beside 15 us a row and CU of arithmetic, two exponentials a logit.  Read
// twice it took 537, kept in registers without the next row's loads between the stores 427.
// Neither nontemporal loads or stores nor statistics 3 or 8 vectors behind the loads change it.
template <typename E, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void policy_rows_kernel(TokenLoss a, PolicyArgs p) {
  __shared__ Stat red[NT / 64 < 1 ? 1 : NT / 64];
  const int nz = (a.V + E::VEC - 1) / E::VEC, nv = (int)(a.ld / E::VEC);
  int tid = threadIdx.x;
  const int off = tid * 16;
  constexpr int LAG = NV < 5 ? NV : 5;
  constexpr int SPAN = NT * E::VEC;  // elements of one vector of every thread
  u32x4 x[NV];
  auto buffer = [&](const void *q, int vecs) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(q), 0, min(vecs, NV * NT) * 16, 0x00020000);
  };
  // The next row from t on of this workgroup with a weight, the others' dz cleared.
  auto next_row = [&](int64_t t) {
    for (; t < a.T && weight(a, t) == 0.0f; t += gridDim.x) {
      if (a.dz) {
        u32x4 *out = dz_ptr<E>(a, t);
        for (int i = tid; i < nv; i += NT) out[i] = zero16();
      }
      if (tid == 0) {
        a.logp[t] = 0.0f;
        a.rows[t] = 0.0f;
      }
    }
    return t;
  };
  int64_t t = next_row(blockIdx.x);
  if (t >= a.T) return;
  auto rs = buffer(row_ptr<E>(a, t), nz);
#pragma unroll
  for (int v = 0; v < NV; ++v) x[v] = __builtin_amdgcn_raw_buffer_load_b128(rs, off, v * NT * 16, 0);
  Stat st{-INFINITY, 0.0f};
  int V = a.V;
  auto take = [&](int v) {  // vector v into the row's statistics
    if (v * SPAN < V) {
      if ((v + 1) * SPAN > V) x[v] = cut_row(E(), x[v], v * NT + tid, V, neg_inf_bits(E()));
      stat_vec<E>(st, x[v]);
    }
    // (the vector stays packed: without this the compiler keeps its elements for dz, and spills)
    asm volatile("" : "+v"(x[v]));
  };
#pragma unroll
  for (int v = 0; v < NV; ++v) take(v);
  while (t < a.T) {
    // (what depends on V and on the thread's columns is recomputed for each row, not kept in registers)
    asm volatile("" : "+s"(V), "+v"(tid));
    const u32x4 *zrow = row_ptr<E>(a, t);
#pragma unroll 4
    for (int i = NV * NT + tid; i < nz; i += NT) {
      u32x4 r = zrow[i];
      if ((i + 1) * E::VEC > V) r = cut_row(E(), r, i, V, neg_inf_bits(E()));
      stat_vec<E>(st, r);
    }
    st = block_stat<NT>(st, red);
    const double logp = logp_of(target_logit<E>(a, t), st);
    float l, g;
    policy_terms(p, t, logp, &l, &g);
    const float w = weight(a, t), c = w * g;
    if (tid == 0) {
      a.logp[t] = (float)logp;
      a.rows[t] = w * l;
    }
    const int64_t tn = next_row(t + gridDim.x);
    rs = buffer(row_ptr<E>(a, tn < a.T ? tn : t), tn < a.T ? nz : 0);
    const float m = st.m, k = -c / st.s;
    const int y = a.y[t];
    st = Stat{-INFINITY, 0.0f};
    if (NT > 64) __syncthreads();  // dz may be z: the target's logit has been read by every wave
    const auto os = buffer(a.dz ? dz_ptr<E>(a, t) : nullptr, a.dz ? nv : 0);
#pragma unroll
    for (int v = 0; v < NV + LAG; ++v) {
      if (v < NV) {
        u32x4 d = zero16();
        if (a.dz && c != 0.0f && v * SPAN < V) {
          d = dz_vec<E>(x[v], v * NT + tid, m, k, c, y);
          if ((v + 1) * SPAN > V) d = cut_row(E(), d, v * NT + tid, V, 0u);
        }
        __builtin_amdgcn_raw_buffer_store_b128(d, os, off, v * NT * 16, 0);
        x[v] = __builtin_amdgcn_raw_buffer_load_b128(rs, off, v * NT * 16, 0);
      }
      if (v >= LAG) take(v - LAG);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (a.dz) {
      u32x4 *out = dz_ptr<E>(a, t);
      int i = NV * NT + tid;
      if (c != 0.0f) {
#pragma unroll 4
        for (; i < nz; i += NT) {
          u32x4 d = dz_vec<E>(zrow[i], i, m, k, c, y);
          if ((i + 1) * E::VEC > V) d = cut_row(E(), d, i, V, 0u);
          out[i] = d;
        }
      }
      for (; i < nv; i += NT) out[i] = zero16();
    }
    t = tn;
  }
}

// Parts of a row in the launches that take few rows: at most a wave's lanes, none under
// 16 KB (of 4, 8, 16 and 32 KB the best over a pair, a short answer and a short rollout).
// Before a gradient: enough for about 8192 workgroups (2048 x 151936 bf16 in pairs 326 us,
// whole rows 370).  Log-probabilities alone, whose parts meet: 2048 workgroups, and rows up to
// 64 KB whole (bf16, whole and in parts for 2048 workgroups: 1024 x 32000 12.9 and 16.0 us, 200
// 6.8 and 8.0, 4 6.4 and 6.2; fp32 4 x 16000 6.2 and 6.6; 512 x 151936 bf16 28.7 in parts, whole rows
// 36.5, 33.3 in parts for 8192).
LossPlan loss_plan(int64_t T, int64_t V, Dtype d, bool logp_only) {
  const int64_t vec = d == DT_BF16 ? 8 : 4, nz = (V + vec - 1) / vec;
  const int64_t want = ((logp_only ? 2048 : 8192) + T - 1) / T;
  int64_t parts = std::min<int64_t>(std::min(want, nz / 1024), 64);
  if (parts < 1 || (logp_only && nz <= 4096)) parts = 1;
  LossPlan p{};
  p.part_vecs = (int)((nz + parts - 1) / parts);
  p.parts = (int)((nz + p.part_vecs - 1) / p.part_vecs);
  return p;
}

template <typename E>
static void logp_launch(const TokenLoss &a, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.T * a.parts));
  if (a.parts > 1) hipLaunchKernelGGL(logp_parts_kernel<E>, grid, dim3(TL_NT), 0, st, a);
  else hipLaunchKernelGGL(token_stat_kernel<E>, grid, dim3(TL_NT), 0, st, a, (Stat *)nullptr);
}
hipError_t launch_token_logp(const TokenLoss &a, Dtype d, hipStream_t st) {
  if (d == DT_BF16) logp_launch<BF16>(a, st);
  else logp_launch<F32>(a, st);
  return hipGetLastError();
}

template <typename E, int NT, int NV>
static void policy_rows(const TokenLoss &a, const PolicyArgs &p, int per_cu, hipStream_t st) {
  const int grid = a.T < 256 * per_cu ? a.T : 256 * per_cu;
  hipLaunchKernelGGL((policy_rows_kernel<E, NT, NV>), dim3(grid), dim3(NT), 0, st, a, p);
}

template <typename E>
static void policy_launches(const TokenLoss &a, const PolicyArgs &p, hipStream_t st) {
  if (a.T < POLICY_ROWS && a.parts > 1) {
    Stat *stat = (Stat *)a.stat;
    hipLaunchKernelGGL(token_stat_kernel<E>, dim3((unsigned)((int64_t)a.T * a.parts)), dim3(TL_NT), 0, st, a, stat);
    hipLaunchKernelGGL(policy_parts_kernel<E>, dim3((unsigned)(a.dz ? (int64_t)a.T * a.parts + LOSS_WGS : 1)), dim3(TL_NT), 0,
                       st, a, p, stat);
    return;
  }
  const int nz = (a.V + E::VEC - 1) / E::VEC;
  if (nz <= 64 * 8) policy_rows<E, 64, 8>(a, p, 16, st);
  else if (nz <= 256 * 8) policy_rows<E, 256, 8>(a, p, 4, st);
  else if (nz <= 256 * 16) policy_rows<E, 256, 16>(a, p, 4, st);
  else if (nz <= 1024 * 8) policy_rows<E, 1024, 8>(a, p, 1, st);
  else if (nz <= 1024 * 16) policy_rows<E, 1024, 16>(a, p, 1, st);
  else policy_rows<E, 1024, 20>(a, p, 1, st);
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(LS_NT), 0, st, a.rows, a.T, 1.0, a.loss);
}

hipError_t launch_policy_loss(const TokenLoss &a, const PolicyArgs &p, Dtype d, hipStream_t st) {
  if (d == DT_BF16) policy_launches<BF16>(a, p, st);
  else policy_launches<F32>(a, p, st);
  return hipGetLastError();
}

template <typename E>
static void pair_launches(const TokenLoss &a, const PairArgs &p, hipStream_t st) {
  Stat *stat = (Stat *)a.stat, *rowstat = stat + (int64_t)a.T * a.parts;
  const dim3 grid((unsigned)((int64_t)a.T * a.parts));
  hipLaunchKernelGGL(token_stat_kernel<E>, grid, dim3(TL_NT), 0, st, a, stat);
  hipLaunchKernelGGL(pair_kernel, dim3(p.pairs), dim3(PR_NT), 0, st, a, p, stat, rowstat);
  // Logits that outgrow the last-level cache (256 MB): dz is kept out of it, for the second
  // read of the logits (2048 x 151936 bf16, 622 MB: statistics and dz 60 + 185 us, else
  // 96 + 178).  Smaller ones: dz stays there for the product that reads it next.
  const dim3 dzgrid(a.dz ? grid.x + 1 : 1);
  if ((int64_t)a.T * a.ld * (16 / E::VEC) > (int64_t)256 << 20)
    hipLaunchKernelGGL((pair_dz_kernel<E, true>), dzgrid, dim3(TL_NT), 0, st, a, rowstat, p.pairs);
  else
    hipLaunchKernelGGL((pair_dz_kernel<E, false>), dzgrid, dim3(TL_NT), 0, st, a, rowstat, p.pairs);
}

hipError_t launch_preference_loss(const TokenLoss &a, const PairArgs &p, Dtype d, hipStream_t st) {
  if (d == DT_BF16) pair_launches<BF16>(a, p, st);
  else pair_launches<F32>(a, p, st);
  return hipGetLastError();
}

}  // namespace lora
