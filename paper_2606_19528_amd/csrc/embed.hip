// embed.hip -- embedding lookup and its gradient.
//   out[t]  = scale table[ids[t]]
//   dE[v]   = scale sum over t with ids[t] = v of dout[t], ascending t
// An id outside [0, V) has a zero output row and no gradient.
//
// The gradient's positions are sorted by token (stable radix sort, so equal
// tokens keep ascending t) and cut into chunks of equally many sorted
// positions: a chunk's work does not depend on how often a token occurs.  A
// chunk sums its tokens' rows one after another in registers.  What it holds
// of a token that began in an earlier chunk goes to its partial sum, and the
// join launch adds a token's partial sums in chunk order: no atomics, one
// order of summation.
#include "kernels.hpp"
#include "launch.hpp"

namespace lora {

// One wave a token.
constexpr int EF_NT = 256;
template <typename E>
__global__ __launch_bounds__(EF_NT) void embed_fwd_kernel(const typename E::T *table, const int32_t *ids,
                                                          typename E::T *out, int T, int V, int vpr, float scale) {
  const int t = blockIdx.x * (EF_NT / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= T) return;
  const int id = __builtin_amdgcn_readfirstlane(ids[t]);
  const bool ok = id >= 0 && id < V;
  const u32x4 *src = (const u32x4 *)table + (int64_t)(ok ? id : 0) * vpr;
  u32x4 *dst = (u32x4 *)out + (int64_t)t * vpr;
  for (int v = lane; v < vpr; v += 64) {
    u32x4 x = zero16();
    if (ok) {
      float f[E::VEC];
      unpack_vec(E(), src[v], f);
#pragma unroll
      for (int e = 0; e < E::VEC; ++e) f[e] *= scale;
      x = pack_vec(E(), f);
    }
    dst[v] = x;
  }
}

// ---- stable radix sort of (token, position) ------------------------------------
// Keys are tokens, V for an id outside [0, V) so that those sort last.  One pass
// per digit of up to 9 bits over tiles of 2048 keys: the tiles' digit counts
// (digit-major), their prefix along the tiles, the scatter.
constexpr int RS_NT = 256, RS_R = 8, RS_TILE = RS_NT * RS_R, RS_BINS = 512, RS_WAVES = RS_NT / 64;

__device__ __forceinline__ uint32_t embed_key(int32_t id, int V) { return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V; }

__global__ __launch_bounds__(RS_NT) void radix_count_kernel(const uint32_t *key, bool ids, int n, int V, int shift, int bins,
                                                            int ntile, int *count) {
  __shared__ int h[RS_BINS];
  for (int d = threadIdx.x; d < bins; d += RS_NT) h[d] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < RS_R; ++r) {
    const int64_t i = (int64_t)blockIdx.x * RS_TILE + r * RS_NT + threadIdx.x;
    if (i < n) {
      const uint32_t k = ids ? embed_key((int32_t)key[i], V) : key[i];
      atomicAdd(&h[(k >> shift) & (bins - 1)], 1);
    }
  }
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += RS_NT) count[(int64_t)d * ntile + blockIdx.x] = h[d];
}

// Inclusive sum over a wave.
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(x, off);
    if (lane >= off) x += y;
  }
  return x;
}
// Exclusive sum over a workgroup of NT threads; *total receives the whole sum.
template <int NT>
__device__ __forceinline__ int block_scan(int x, int *part, int *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int inc = wave_scan(x, lane);
  __syncthreads();
  if (lane == 63) part[wave] = inc;
  __syncthreads();
  int base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wave) base += part[w];
    all += part[w];
  }
  *total = all;
  return base + inc - x;
}

// One workgroup a digit: its counts become their exclusive prefix along the tiles.
__global__ __launch_bounds__(RS_NT) void radix_prefix_kernel(int *count, int ntile, int *total) {
  __shared__ int part[RS_WAVES];
  int *row = count + (int64_t)blockIdx.x * ntile;
  int base = 0;
  for (int t0 = 0; t0 < ntile; t0 += RS_NT) {
    const int t = t0 + threadIdx.x;
    int all;
    const int x = t < ntile ? row[t] : 0;
    const int e = block_scan<RS_NT>(x, part, &all);
    if (t < ntile) row[t] = base + e;
    base += all;
  }
  if (threadIdx.x == 0) total[blockIdx.x] = base;
}

// A wave owns 512 consecutive keys, 64 a round; lanes with equal digits find
// each other by ballots, so a key's rank among its wave's equal digits is the
// count of the earlier rounds plus the lower lanes of its own.
__global__ __launch_bounds__(RS_NT) void radix_scatter_kernel(const uint32_t *key, const int32_t *pos, bool ids, int n, int V,
                                                              int shift, int bits, int ntile, const int *count, const int *total,
                                                              uint32_t *key_out, int32_t *pos_out) {
  __shared__ int cnt[RS_WAVES][RS_BINS];
  __shared__ int base[RS_BINS];
  __shared__ int part[RS_WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << bits;
  for (int d = threadIdx.x; d < RS_WAVES * RS_BINS; d += RS_NT) (&cnt[0][0])[d] = 0;
  int run = 0;
  for (int d0 = 0; d0 < bins; d0 += RS_NT) {  // keys of smaller digits, and of this digit in earlier tiles
    const int d = d0 + threadIdx.x;
    int all;
    const int x = d < bins ? total[d] : 0;
    const int e = block_scan<RS_NT>(x, part, &all);
    if (d < bins) base[d] = run + e + count[(int64_t)d * ntile + blockIdx.x];
    run += all;
  }
  __syncthreads();
  uint32_t k[RS_R];
  int rank[RS_R];
  const int64_t i0 = (int64_t)blockIdx.x * RS_TILE + wave * 64 * RS_R + lane;
#pragma unroll
  for (int r = 0; r < RS_R; ++r) {
    const int64_t i = i0 + r * 64;
    k[r] = 0;
    if (i < n) k[r] = ids ? embed_key((int32_t)key[i], V) : key[i];
  }
#pragma unroll
  for (int r = 0; r < RS_R; ++r) {
    const bool in = i0 + r * 64 < n;
    const int d = (k[r] >> shift) & (bins - 1);
    uint64_t peers = __ballot(in);
    for (int b = 0; b < bits; ++b) {
      const bool one = (d >> b) & 1;
      const uint64_t m = __ballot(one);
      peers &= one ? m : ~m;
    }
    const uint64_t below = peers & ((1ull << lane) - 1ull);
    const int before = cnt[wave][d];
    rank[r] = before + __popcll(below);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in && below == 0) cnt[wave][d] = before + __popcll(peers);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += RS_NT) {
    int s = base[d];
#pragma unroll
    for (int w = 0; w < RS_WAVES; ++w) {
      const int c = cnt[w][d];
      cnt[w][d] = s;
      s += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < RS_R; ++r) {
    const int64_t i = i0 + r * 64;
    if (i >= n) continue;
    const int o = cnt[wave][(k[r] >> shift) & (bins - 1)] + rank[r];
    key_out[o] = k[r];
    pos_out[o] = pos ? pos[i] : (int32_t)i;
  }
}

// ---- numbers of the distinct tokens ----------------------------------------------
// A sorted place is a head when its token is in range and differs from the one
// before; seg[i] = number of the place's token among the distinct ones.
constexpr int SG_NT = 256, SG_R = 8, SG_TILE = SG_NT * SG_R;

__device__ __forceinline__ bool is_head(const uint32_t *sid, int64_t i, int n, int V) {
  return i < n && sid[i] != (uint32_t)V && (i == 0 || sid[i - 1] != sid[i]);
}
__global__ __launch_bounds__(SG_NT) void seg_count_kernel(const uint32_t *sid, int n, int V, int *count) {
  __shared__ int part[SG_NT / 64];
  int c = 0;
  for (int r = 0; r < SG_R; ++r)
    c += is_head(sid, (int64_t)blockIdx.x * SG_TILE + r * SG_NT + threadIdx.x, n, V);
  int all;
  block_scan<SG_NT>(c, part, &all);
  if (threadIdx.x == 0) count[blockIdx.x] = all;
}
// count becomes its exclusive prefix, total[0] the number of distinct tokens.
__global__ __launch_bounds__(SG_NT) void seg_kernel(const uint32_t *sid, int n, int V, const int *before, int *seg, int32_t *tokens) {
  __shared__ int part[SG_NT / 64];
  int run = before[blockIdx.x] - 1;
  for (int r = 0; r < SG_R; ++r) {
    const int64_t i = (int64_t)blockIdx.x * SG_TILE + r * SG_NT + threadIdx.x;
    const bool h = is_head(sid, i, n, V);
    int all;
    const int e = block_scan<SG_NT>(h, part, &all);
    if (i < n) {
      const int s = run + e + (h ? 1 : 0);
      seg[i] = s;
      if (h) tokens[s] = (int32_t)sid[i];
    }
    run += all;
  }
}

// ---- sums ---------------------------------------------------------------------------
constexpr int EG_NT = 128, EG_U = 8;

struct EmbedGrad {
  const uint32_t *sid;   // [T] sorted tokens (V: none)
  const int32_t *order;  // [T] their positions
  const int *seg;        // [T] numbers of distinct tokens, and
  const int *nseg;       //     how many there are (compact form)
  const void *dout;
  float *out;            // [V][D], or compact [cap][D]
  int32_t *tokens;       // compact form, [cap]; else null
  float *partial;        // [chunks][D]
  int T, V, D, cap, chunk, nchunk, ncol, accumulate;
  float scale;
};

__device__ __forceinline__ int64_t grad_row(const EmbedGrad &a, int64_t i) { return a.tokens ? a.seg[i] : (int64_t)a.sid[i]; }

template <typename E>
__device__ __forceinline__ void put_grad(const EmbedGrad &a, int64_t row, int v, const float *acc, bool add) {
  float *o = a.out + row * a.D + v * E::VEC;
#pragma unroll
  for (int q = 0; q < E::VEC / 4; ++q) {
    f32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a.scale * acc[4 * q + e];
    if (add) x += ((const f32x4 *)o)[q];
    ((f32x4 *)o)[q] = x;
  }
}

// Workgroups [0, nchunk * ncol): a chunk and a block of EG_NT vectors of its
// columns each.  The rest clear what no token reaches: 64 rows each.
template <typename E>
__global__ __launch_bounds__(EG_NT) void embed_grad_kernel(EmbedGrad a) {
  const int vpr = a.D / E::VEC;
  const unsigned work = (unsigned)a.nchunk * a.ncol;
  if (blockIdx.x >= work) {
    const int64_t r0 = (int64_t)(blockIdx.x - work) * 64;
    const int lane = threadIdx.x & 63;
    const int64_t rows = a.tokens ? a.cap : a.V;
    const int64_t r = r0 + lane;
    bool used = r >= rows;
    if (a.tokens) used = used || r < a.nseg[0];
    else if (!used) {  // lower bound of token r among the sorted ones
      int lo = 0, hi = a.T;
      while (lo < hi) {
        const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);
        if (a.sid[mid] < (uint32_t)r) lo = mid + 1;
        else hi = mid;
      }
      used = lo < a.T && a.sid[lo] == (uint32_t)r;
    }
    uint64_t clear = ~__ballot(used);
    if (a.tokens && threadIdx.x < 64 && !used) a.tokens[r] = -1;
    while (clear) {
      const int l = __ffsll((unsigned long long)clear) - 1;
      clear &= clear - 1;
      f32x4 *o = (f32x4 *)(a.out + (r0 + l) * a.D);
      for (int v = threadIdx.x; v < a.D / 4; v += EG_NT) o[v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    return;
  }
  const int chunk = blockIdx.x / a.ncol, v = (blockIdx.x % a.ncol) * EG_NT + threadIdx.x;
  if (v >= vpr) return;
  const int64_t c0 = (int64_t)chunk * a.chunk, c1 = min((int64_t)a.T, c0 + a.chunk);
  uint32_t cur = a.sid[c0];
  bool later = c0 > 0 && a.sid[c0 - 1] == cur;  // the token began in an earlier chunk
  int64_t head = c0;
  float acc[E::VEC];
#pragma unroll
  for (int e = 0; e < E::VEC; ++e) acc[e] = 0.0f;
  auto flush = [&]() {
    if (cur == (uint32_t)a.V) return;
    if (later) {
      float *p = a.partial + (int64_t)chunk * a.D + v * E::VEC;
#pragma unroll
      for (int q = 0; q < E::VEC / 4; ++q) ((f32x4 *)p)[q] = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    } else {
      put_grad<E>(a, grad_row(a, head), v, acc, a.accumulate);
    }
  };
  for (int64_t i0 = c0; i0 < c1; i0 += EG_U) {
    u32x4 x[EG_U];
#pragma unroll
    for (int u = 0; u < EG_U; ++u)
      if (i0 + u < c1) x[u] = ((const u32x4 *)a.dout)[(int64_t)a.order[i0 + u] * vpr + v];
#pragma unroll
    for (int u = 0; u < EG_U; ++u) {
      if (i0 + u >= c1) break;
      const uint32_t s = a.sid[i0 + u];
      if (s != cur) {
        flush();
        cur = s;
        later = false;
        head = i0 + u;
#pragma unroll
        for (int e = 0; e < E::VEC; ++e) acc[e] = 0.0f;
      }
      float f[E::VEC];
      unpack_vec(E(), x[u], f);
#pragma unroll
      for (int e = 0; e < E::VEC; ++e) acc[e] += f[e];
    }
  }
  flush();
}

// A token's partial sums, added to its row in chunk order by the workgroups of
// the first chunk that the token runs into.
template <typename E>
__global__ __launch_bounds__(EG_NT) void embed_join_kernel(EmbedGrad a) {
  const int vpr = a.D / E::VEC;
  const int chunk = blockIdx.x / a.ncol + 1, v = (blockIdx.x % a.ncol) * EG_NT + threadIdx.x;
  if (v >= vpr) return;
  const int64_t c0 = (int64_t)chunk * a.chunk;
  const uint32_t tok = a.sid[c0];
  if (tok == (uint32_t)a.V || a.sid[c0 - 1] != tok) return;
  const int64_t b0 = c0 - a.chunk;
  if (b0 > 0 && a.sid[b0] == tok && a.sid[b0 - 1] == tok) return;  // the chunk before it holds a partial sum too
  float acc[E::VEC];
#pragma unroll
  for (int e = 0; e < E::VEC; ++e) acc[e] = 0.0f;
  for (int c = chunk; c < a.nchunk && a.sid[(int64_t)c * a.chunk] == tok; ++c) {
    const float *p = a.partial + (int64_t)c * a.D + v * E::VEC;
#pragma unroll
    for (int e = 0; e < E::VEC; ++e) acc[e] += p[e];
  }
  put_grad<E>(a, grad_row(a, c0), v, acc, true);
}

hipError_t launch_embed_fwd(const void *table, const int32_t *ids, void *out, int T, int V, int D, float scale, Dtype d,
                            hipStream_t st) {
  const dim3 grid((T + EF_NT / 64 - 1) / (EF_NT / 64));
  if (d == DT_BF16)
    hipLaunchKernelGGL(embed_fwd_kernel<BF16>, grid, dim3(EF_NT), 0, st, (const uint16_t *)table, ids, (uint16_t *)out, T, V,
                       D / 8, scale);
  else
    hipLaunchKernelGGL(embed_fwd_kernel<F32>, grid, dim3(EF_NT), 0, st, (const float *)table, ids, (float *)out, T, V, D / 4,
                       scale);
  return hipGetLastError();
}

static size_t up256(size_t b) { return (b + 255) & ~size_t(255); }

EmbedPlan embed_plan(int64_t T, int64_t V, int64_t D) {
  EmbedPlan p{};
  int bits = 1;
  while (((int64_t)1 << bits) <= V) ++bits;  // keys 0 .. V
  p.passes = (bits + 8) / 9;
  p.digit = (bits + p.passes - 1) / p.passes;
  p.ntile = (int)((T + RS_TILE - 1) / RS_TILE);
  p.chunk = T <= 8192 ? EG_U : 4 * EG_U;
  p.nchunk = (int)((T + p.chunk - 1) / p.chunk);
  const int64_t nsg = (T + SG_TILE - 1) / SG_TILE;
  size_t off = 0;
  for (int i = 0; i < 2; ++i) {
    p.key[i] = off;
    off += up256((size_t)T * 4);
    p.pos[i] = off;
    off += up256((size_t)T * 4);
  }
  p.seg = off;
  off += up256((size_t)T * 4);
  p.segcount = off;
  off += up256((size_t)(nsg + 1) * 4);
  p.count = off;
  off += up256(((size_t)p.ntile + 1) * RS_BINS * 4);
  p.partial = off;
  off += up256((size_t)p.nchunk * D * 4);
  p.total = off;
  return p;
}

hipError_t launch_embed_sort(const int32_t *ids, int T, int V, const EmbedPlan &p, char *ws, int32_t *tokens, hipStream_t st) {
  const int bins = 1 << p.digit;
  int *count = (int *)(ws + p.count), *total = count + (int64_t)RS_BINS * p.ntile;
  const uint32_t *key = (const uint32_t *)ids;
  const int32_t *pos = nullptr;
  for (int s = 0; s < p.passes; ++s) {
    const int o = (p.passes - 1 - s) & 1;  // the last pass writes buffer 0
    const bool first = s == 0;
    hipLaunchKernelGGL(radix_count_kernel, dim3(p.ntile), dim3(RS_NT), 0, st, key, first, T, V, s * p.digit, bins, p.ntile,
                       count);
    hipLaunchKernelGGL(radix_prefix_kernel, dim3(bins), dim3(RS_NT), 0, st, count, p.ntile, total);
    hipLaunchKernelGGL(radix_scatter_kernel, dim3(p.ntile), dim3(RS_NT), 0, st, key, pos, first, T, V, s * p.digit, p.digit,
                       p.ntile, count, total, (uint32_t *)(ws + p.key[o]), (int32_t *)(ws + p.pos[o]));
    key = (const uint32_t *)(ws + p.key[o]);
    pos = (const int32_t *)(ws + p.pos[o]);
  }
  if (tokens) {
    const int nsg = (T + SG_TILE - 1) / SG_TILE;
    int *sc = (int *)(ws + p.segcount);
    hipLaunchKernelGGL(seg_count_kernel, dim3(nsg), dim3(SG_NT), 0, st, key, T, V, sc);
    hipLaunchKernelGGL(radix_prefix_kernel, dim3(1), dim3(RS_NT), 0, st, sc, nsg, sc + nsg);
    hipLaunchKernelGGL(seg_kernel, dim3(nsg), dim3(SG_NT), 0, st, key, T, V, sc, (int *)(ws + p.seg), tokens);
  }
  return hipGetLastError();
}

hipError_t launch_embed_grad(const void *dout, float *out, int32_t *tokens, int T, int V, int D, float scale, bool accumulate,
                             Dtype d, const EmbedPlan &p, char *ws, hipStream_t st) {
  EmbedGrad a{};
  a.sid = (const uint32_t *)(ws + p.key[0]);
  a.order = (const int32_t *)(ws + p.pos[0]);
  a.seg = (const int *)(ws + p.seg);
  a.nseg = (const int *)(ws + p.segcount) + (T + SG_TILE - 1) / SG_TILE;
  a.dout = dout;
  a.out = out;
  a.tokens = tokens;
  a.partial = (float *)(ws + p.partial);
  a.T = T;
  a.V = V;
  a.D = D;
  a.cap = T < V ? T : V;
  a.chunk = p.chunk;
  a.nchunk = p.nchunk;
  a.accumulate = accumulate;
  a.scale = scale;
  const int vec = d == DT_BF16 ? 8 : 4;
  a.ncol = (D / vec + EG_NT - 1) / EG_NT;
  const int64_t clear = accumulate ? 0 : ((tokens ? (int64_t)a.cap : (int64_t)V) + 63) / 64;
  const dim3 grid((unsigned)((int64_t)a.nchunk * a.ncol + clear)), join((unsigned)((int64_t)(a.nchunk - 1) * a.ncol));
  if (d == DT_BF16) {
    hipLaunchKernelGGL(embed_grad_kernel<BF16>, grid, dim3(EG_NT), 0, st, a);
    if (a.nchunk > 1) hipLaunchKernelGGL(embed_join_kernel<BF16>, join, dim3(EG_NT), 0, st, a);
  } else {
    hipLaunchKernelGGL(embed_grad_kernel<F32>, grid, dim3(EG_NT), 0, st, a);
    if (a.nchunk > 1) hipLaunchKernelGGL(embed_join_kernel<F32>, join, dim3(EG_NT), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace lora
