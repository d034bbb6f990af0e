// embed.hip -- embedding lookup and its gradient.
//   out[t]  = scale table[ids[t]]
//   dE[v]   = scale sum over t with ids[t] = v of dout[t], ascending t
// An id outside [0, V) has a zero output row and no gradient.
//
// The gradient of many positions (EmbedPlan::scan false): they are sorted by
// token (stable radix sort, so equal tokens keep ascending t) and cut into
// chunks of equally many sorted positions: a chunk's work does not depend on
// how often a token occurs.  A chunk sums its tokens' rows one after another in
// registers.  What it holds of a token that began in an earlier chunk goes to
// its partial sum, and the join launch adds a token's partial sums in chunk
// order, one after another, so that launch's time does depend on the most frequent
// token: no atomics on values, one order of summation for given ids.
//
// The gradient of few positions: six to nine launches of a sort would take
// longer than the sums.  A workgroup instead looks for its positions' tokens
// among all of them: see embed_scan_kernel.
#include <algorithm>

#include "kernels.hpp"
#include "launch.hpp"

namespace lora {

// A wave takes up to 4 vectors a lane of one token's row, all loads before the first
// store.  Bound by memory: 16384 rows of 2048 bf16 18 us (67 MB written, 30 MB of distinct
// rows read: 5.4 TB/s); 24 rows of 3072 2.8 us, 3.5 with a wave a row and a load at a time.
constexpr int EF_NT = 256, EF_U = 4;
template <typename E>
__global__ __launch_bounds__(EF_NT) void embed_fwd_kernel(const typename E::T *table, const int32_t *ids,
                                                          typename E::T *out, int T, int V, int vpr, unsigned per_row,
                                                          float scale) {
  const unsigned w = blockIdx.x * (EF_NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const unsigned t = w / per_row;
  if (t >= (unsigned)T) return;
  const int v0 = (w % per_row) * 64 * EF_U + lane;
  const int id = __builtin_amdgcn_readfirstlane(ids[t]);
  const bool ok = id >= 0 && id < V;
  const u32x4 *src = (const u32x4 *)table + (int64_t)(ok ? id : 0) * vpr;
  u32x4 *dst = (u32x4 *)out + (int64_t)t * vpr, x[EF_U];
#pragma unroll
  for (int u = 0; u < EF_U; ++u) x[u] = ok && v0 + u * 64 < vpr ? src[v0 + u * 64] : zero16();
#pragma unroll
  for (int u = 0; u < EF_U; ++u) {
    if (v0 + u * 64 >= vpr) break;
    float f[E::VEC];
    unpack_vec(E(), x[u], f);
#pragma unroll
    for (int e = 0; e < E::VEC; ++e) f[e] *= scale;
    dst[v0 + u * 64] = ok ? pack_vec(E(), f) : zero16();
  }
}

// ---- stable radix sort of (token, position) ------------------------------------
// Keys are tokens, V for an id outside [0, V) so that those sort last.  One pass
// per digit of up to 9 bits over tiles of 1024 keys: the tiles' digit counts
// (digit-major), their prefix along the tiles, the scatter.  Up to RS_DIRECT
// tiles the scatter sums the counts itself and the prefix launch is spared.
constexpr int RS_DIRECT = 64;
constexpr int RS_NT = 256, RS_R = 4, RS_TILE = RS_NT * RS_R, RS_BINS = 512, RS_WAVES = RS_NT / 64;

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

// A wave owns 64 RS_R consecutive keys, 64 a round; lanes with equal digits find
// each other by ballots, so a key's rank among its wave's equal digits is the
// count of the earlier rounds plus the lower lanes of its own.
__global__ __launch_bounds__(RS_NT) void radix_scatter_kernel(const uint32_t *key, const int32_t *pos, bool ids, int n, int V,
                                                              int shift, int bits, int ntile, const int *count, const int *total,
                                                              bool direct, uint32_t *key_out, int32_t *pos_out) {
  __shared__ int cnt[RS_WAVES][RS_BINS];
  __shared__ int base[RS_BINS];
  __shared__ int part[RS_WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << bits;
  for (int d = threadIdx.x; d < RS_WAVES * RS_BINS; d += RS_NT) (&cnt[0][0])[d] = 0;
  int run = 0;
  for (int d0 = 0; d0 < bins; d0 += RS_NT) {  // keys of smaller digits, and of this digit in earlier tiles
    const int d = d0 + threadIdx.x;
    int all, x = 0, before = 0;
    if (d < bins) {
      const int *row = count + (int64_t)d * ntile;
      if (direct) {
#pragma unroll 8
        for (int t = 0; t < ntile; ++t) {
          x += row[t];
          before += t < (int)blockIdx.x ? row[t] : 0;
        }
      } else {
        x = total[d];
        before = row[blockIdx.x];
      }
    }
    const int e = block_scan<RS_NT>(x, part, &all);
    if (d < bins) base[d] = run + e + before;
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
constexpr int SG_OWN = 16;  // tiles up to which each counts the heads before it itself

// Heads among the places i .. i + 7 (i a multiple of 8), as bits.
__device__ __forceinline__ uint32_t heads8(const uint32_t *sid, int64_t i, int n, int V, uint32_t *k) {
  if (i >= n) return 0;
  uint32_t last = i > 0 ? sid[i - 1] : (uint32_t)V;
  if (i + 8 <= n) {
    const u32x4 lo = ld16(sid + i), hi = ld16(sid + i + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      k[e] = lo[e];
      k[4 + e] = hi[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = i + e < n ? sid[i + e] : (uint32_t)V;
  }
  uint32_t h = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    h |= (uint32_t)(k[e] != (uint32_t)V && k[e] != last) << e;
    last = k[e];
  }
  return h;
}
__global__ __launch_bounds__(SG_NT) void seg_count_kernel(const uint32_t *sid, int n, int V, int *count) {
  __shared__ int part[SG_NT / 64];
  uint32_t k[SG_R];
  int all;
  block_scan<SG_NT>(__popc(heads8(sid, (int64_t)blockIdx.x * SG_TILE + threadIdx.x * SG_R, n, V, k)), part, &all);
  if (threadIdx.x == 0) count[blockIdx.x] = all;
}
// before: heads ahead of each tile (and behind them the number of heads in all); null:
// each workgroup counts them itself, and the last one leaves the number in nseg.
__global__ __launch_bounds__(SG_NT) void seg_kernel(const uint32_t *sid, int n, int V, const int *before, int *nseg, int *seg,
                                                    int32_t *tokens) {
  __shared__ int part[SG_NT / 64];
  uint32_t k[SG_R];
  const int64_t i0 = (int64_t)blockIdx.x * SG_TILE + threadIdx.x * SG_R;
  int run = -1, all;
  if (before) {
    run += before[blockIdx.x];
  } else {
    int c = 0;
#pragma unroll 4
    for (int b = 0; b < (int)blockIdx.x; ++b) c += __popc(heads8(sid, (int64_t)b * SG_TILE + threadIdx.x * SG_R, n, V, k));
    block_scan<SG_NT>(c, part, &all);
    run += all;
  }
  const uint32_t h = heads8(sid, i0, n, V, k);
  run += block_scan<SG_NT>(__popc(h), part, &all);
#pragma unroll
  for (int e = 0; e < SG_R; ++e) {
    if (i0 + e >= n) break;
    if ((h >> e) & 1u) tokens[++run] = (int32_t)k[e];
    seg[i0 + e] = run;
  }
  if (!before && blockIdx.x == gridDim.x - 1 && threadIdx.x == SG_NT - 1) nseg[0] = run + 1;
}

// ---- clearing ------------------------------------------------------------------------
// One vector a thread: 1.2 GB at 6.8 TB/s.  (Four a thread 6.1; loops of 256 workgroups of
// 256 threads side by side 6.5, and 5.2 with a look at a bitmap of the tokens present, so that
// no row is written twice; 64 rows a workgroup 5.3.)
constexpr int CL_NT = 256;
__global__ __launch_bounds__(CL_NT) void clear_kernel(f32x4 *out, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * CL_NT + threadIdx.x;
  if (i < n) out[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
}
static void clear(float *out, int64_t rows, int64_t D, hipStream_t st) {
  constexpr int64_t most = (int64_t)1 << 30;  // vectors a launch
  for (int64_t v0 = 0, n = rows * (D / 4); v0 < n; v0 += most)
    hipLaunchKernelGGL(clear_kernel, dim3((unsigned)((std::min(most, n - v0) + CL_NT - 1) / CL_NT)), dim3(CL_NT), 0, st,
                       (f32x4 *)out + v0, std::min(most, n - v0));
}

// ---- sums ---------------------------------------------------------------------------
// 16384 positions of 151936 x 2048: sort 24 us, numbers 7, sums 37, join 9 (201 MB, 39 us at a
// copy's rate, and in the last-level cache); of 128256 x 3072 the sums alone take 78 (300 MB, 59).
constexpr int EG_NT = 256, EG_COL = 128, EG_U = 8;  // a workgroup: two chunks by EG_COL vectors

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

// Workgroups [0, nwork): two chunks and a block of EG_COL vectors of their columns
// each.  Compact form: the rest clear 64 rows each of those that no token reaches.
template <typename E>
__global__ __launch_bounds__(EG_NT) void embed_grad_kernel(EmbedGrad a, unsigned nwork) {
  const int vpr = a.D / E::VEC;
  if (blockIdx.x >= nwork) {
    const int64_t r0 = (int64_t)(blockIdx.x - nwork) * 64, r1 = min(r0 + 64, (int64_t)a.cap);
    for (int64_t r = max(r0, (int64_t)a.nseg[0]); r < r1; ++r) {
      if (threadIdx.x == 0) a.tokens[r] = -1;
      f32x4 *o = (f32x4 *)(a.out + r * a.D);
      for (int v = threadIdx.x; v < a.D / 4; v += EG_NT) o[v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    return;
  }
  const int chunk = blockIdx.x / a.ncol * 2 + threadIdx.x / EG_COL, v = (blockIdx.x % a.ncol) * EG_COL + threadIdx.x % EG_COL;
  if (v >= vpr || chunk >= a.nchunk) return;
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
// the first chunk that the token runs into.  Bound by that chain, a chunk's key and then its
// sum, where a token is frequent: 32768 positions of 151936 x 2048 compact take 153 us with
// a text's frequencies, 345 with half of them one token (512 chunks), 548 with all.
template <typename E>
__global__ __launch_bounds__(EG_COL) void embed_join_kernel(EmbedGrad a) {
  const int vpr = a.D / E::VEC;
  const int chunk = blockIdx.x / a.ncol + 1, v = (blockIdx.x % a.ncol) * EG_COL + threadIdx.x;
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

// ---- few positions: no sort ------------------------------------------------------------
// The occurrences of a token, in ascending t, are cut into runs of RUN, and the
// rows of a run are summed by the workgroup of the position that starts it.  The
// first run's sum is the token's row; a later run's goes to a slot of its own,
// and the join launch adds the slots of a token.
// A workgroup of W waves takes W positions.  Each wave holds a W-th of all T tokens
// in registers and compares it with the workgroup's W tokens (ballots): how
// many equal ones lie before a position, and which are the next after it.
// Slots: with L smaller tokens among the positions, run i of a token takes slot
// (L + RUN i) / RUN, i > 0: in sorted order RUN positions of the same token lie
// before it, so no other run's quotient is the same.
// The compact form's row of a token is its rank in a bitmap of all tokens
// present, which every workgroup builds in LDS.
// 4096 positions of 128256 x 3072, frequencies of a text: 27 us and 7 for the join (75 MB, 15 us
// at a copy's rate).  At 64 columns 18 remain, a chain in each workgroup: loads 0.6, bitmap and
// its counts 4, comparisons 3, joins 2, rows 3.  More positions a workgroup (8 instead of 4: 37
// us in all for 34, and 24 against 20 at 512 positions) lengthen it.
constexpr int ES_RUN = 8, ES_BATCH = 8;  // rows of a run, and of those that a thread loads at once
constexpr int ES_COLS = 256;  // columns of an item of the join launch
// Up to this many positions a run holds all of a token's, and one launch does.  32 distinct
// tokens: 11.9 us for 14.6 with the second launch (3072 columns), 15.4 for 18.0 (8192); four
// tokens 8 times each 16.5 for 19.2 and 23.7 for 26.5.  One token 32 times, in a workgroup
// alone, loses: 17.6 for 15.4 and 30.8 for 17.7.  At 64 the repeated ones lose more (four
// tokens 16 times 54.7 for 30.4) than distinct ones gain.
constexpr int ES_FEW = 32;
// Rows that a workgroup of the dense form clears, a bit each: 14913 x 1392 15.5 us, 64 rows 18.0;
// 16 and 8 alike, but 8192 positions of 50257 x 768 take 39.9, 41.5 and 49.4.
constexpr int ES_CLEAR = 32;
constexpr int ES_U = 4;  // a lane holds 4 ES_U tokens: T <= 16 NT

struct EmbedScan {
  const int32_t *ids;
  const void *dout;
  float *out;
  int32_t *tokens;  // compact form; else null
  // workspace: slots [T / RUN + 1][D]; per workgroup the number of its tokens with
  // more than one run, and for each its row, first slot and number of slots
  float *slots;
  int32_t *nhot, *hot;
  int T, V, D, cap, nwg, accumulate;
  float scale;
};

// Four elements of a row.
__device__ __forceinline__ f32x4 row4(BF16, const void *row, int v) {
  const uint2 x = ((const uint2 *)row)[v];
  return f32x4{__builtin_bit_cast(float, x.x << 16), __builtin_bit_cast(float, x.x & 0xffff0000u),
               __builtin_bit_cast(float, x.y << 16), __builtin_bit_cast(float, x.y & 0xffff0000u)};
}
__device__ __forceinline__ f32x4 row4(F32, const void *row, int v) { return ((const f32x4 *)row)[v]; }

// Positions base + 4 lane .. + 3 of the ids; -1 past the end.
__device__ __forceinline__ int4 ids4(const int32_t *ids, int base, int lane, int T) {
  const int i = base + 4 * lane;
  if (i + 4 <= T) return *(const int4 *)(ids + i);
  int4 k;
  k.x = i < T ? ids[i] : -1;
  k.y = i + 1 < T ? ids[i + 1] : -1;
  k.z = i + 2 < T ? ids[i + 2] : -1;
  k.w = -1;
  return k;
}
// Lanes whose position base + 4 lane + c is below t.
__device__ __forceinline__ uint64_t lanes_below(int t, int base, int c) {
  const int n = (t - base - c + 3) >> 2;
  return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull;
}
__device__ __forceinline__ int below_lane(uint64_t m) {  // bits of m below this lane
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// Sum of the rows of positions t, list[0 .. n), n < R, into the row `dst`, by NT
// threads.  All R rows are loaded, so that no branch stands between the loads
// of several columns; those past n are the first row again.
template <typename E, int NT, int R>
__device__ __forceinline__ void sum_rows(const EmbedScan &a, int t, const int *list, int n, float *dst, float scale, bool add) {
  const int64_t bytes = (int64_t)a.D * sizeof(typename E::T);
  const char *x = (const char *)a.dout;
  const int nv = a.D / 4;
  const char *row[R];
  row[0] = x + t * bytes;
#pragma unroll
  for (int u = 1; u < R; ++u) row[u] = x + (int64_t)(u <= n ? __builtin_amdgcn_readfirstlane(list[u - 1]) : t) * bytes;
#pragma unroll(R < 4 ? 8 : 2)
  for (int v = threadIdx.x & (NT - 1); v < nv; v += NT) {
    f32x4 f[R];
#pragma unroll
    for (int u = 0; u < R; ++u) f[u] = row4(E(), row[u], v);
#pragma unroll
    for (int u = 1; u < R; ++u) f[0] += u <= n ? f[u] : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 s = f[0] * scale, *o = (f32x4 *)dst + v;
    *o = add ? s + *o : s;
  }
}
// The same for more rows, ES_BATCH at a time.
template <typename E, int NT>
__device__ __forceinline__ void sum_long(const EmbedScan &a, int t, const int *list, int n, float *dst, float scale, bool add) {
  const int64_t bytes = (int64_t)a.D * sizeof(typename E::T);
  const char *x = (const char *)a.dout;
  for (int v = threadIdx.x & (NT - 1); v < a.D / 4; v += NT) {
    f32x4 s = row4(E(), x + t * bytes, v);
    for (int b = 0; b < n; b += ES_BATCH) {
      f32x4 f[ES_BATCH];
#pragma unroll
      for (int u = 0; u < ES_BATCH; ++u)
        f[u] = row4(E(), x + (int64_t)__builtin_amdgcn_readfirstlane(list[min(b + u, n - 1)]) * bytes, v);
#pragma unroll
      for (int u = 0; u < ES_BATCH; ++u) s += b + u < n ? f[u] : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    s *= scale;
    f32x4 *o = (f32x4 *)dst + v;
    *o = add ? s + *o : s;
  }
}

// RUN is ES_RUN, or ES_FEW for T <= ES_FEW, where no token has a second run.
template <typename E, int NT, int RUN>
__global__ __launch_bounds__(NT) void embed_scan_kernel(EmbedScan a) {
  constexpr int W = NT / 64;
  extern __shared__ uint32_t lds[];  // compact form: bitmap words
  __shared__ int stretch[NT];        // and the marks before each thread's
  __shared__ int near[W][W][RUN];  // of position q, as wave w sees it: the next occurrences in its part,
  __shared__ int nnear[W][W], nbefore[W][W];  // how many of them, how many before q
  __shared__ int nless[W][W], nequal[W][W];
  __shared__ int list[W][RUN];
  __shared__ int run[W][3];  // 1: the token's row, 2: a slot, 0: none; its number; rows after the first
  __shared__ int hot[W][3], again[W];
  __shared__ int part[W];
  // (the wave's number is read into a scalar, so that what hangs on it stays in scalar registers)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x >= a.nwg) {  // dense form, not cleared ahead: the rows of ES_CLEAR tokens that do not occur
    const int r0 = (int)(blockIdx.x - a.nwg) * ES_CLEAR;
    if (threadIdx.x == 0) lds[0] = 0;
    __syncthreads();
    for (int i = threadIdx.x * 4; i < a.T; i += NT * 4) {
      const int4 k = ids4(a.ids, i - 4 * lane, lane, a.T);
      const int kk[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (kk[c] >= r0 && kk[c] - r0 < ES_CLEAR) atomicOr(&lds[0], 1u << (kk[c] - r0));
    }
    __syncthreads();
    const uint32_t mask = lds[0];
    const int rows = min(ES_CLEAR, a.V - r0);
    for (int r = wave; r < rows; r += W) {
      if ((mask >> r) & 1u) continue;
      f32x4 *o = (f32x4 *)(a.out + (int64_t)(r0 + r) * a.D);
      for (int v = lane; v < a.D / 4; v += 64) o[v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    return;
  }
  // This wave's part of the tokens: ES_U groups of 256 positions from p0 on.
  const int groups = ((a.T + 255) / 256 + W - 1) / W, p0 = wave * groups * 256;
  int4 x[ES_U];
#pragma unroll
  for (int u = 0; u < ES_U; ++u) x[u] = u < groups ? ids4(a.ids, p0 + u * 256, lane, a.T) : int4{-1, -1, -1, -1};
  const int t0 = blockIdx.x * W;
  int ks = lane < W && t0 + lane < a.T ? a.ids[t0 + lane] : -1;  // lane q: the workgroup's token q, -1: none
  if (ks >= a.V || ks < 0) ks = -1;
  const int words = (a.V + 31) / 32;
  if (a.tokens) {
    for (int i = threadIdx.x; i < words; i += NT) lds[i] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < ES_U; ++u) {
      const int kk[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      uint32_t seen[4];  // (most of a frequent token's marks find it marked)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        seen[c] = kk[c] >= 0 && kk[c] < a.V ? ((volatile uint32_t *)lds)[kk[c] >> 5] >> (kk[c] & 31) & 1u : 1u;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (!seen[c]) atomicOr(&lds[kk[c] >> 5], 1u << (kk[c] & 31));
    }
  }
  // Occurrences before each position, in this wave's part.  (The loops over positions are
  // not unrolled: a launch runs the code once, so its length is time.)
#pragma unroll 1
  for (int q = 0; q < W; ++q) {
    const int t = t0 + q, k = __builtin_amdgcn_readlane(ks, q);
    int nb = 0;
#pragma unroll
    for (int u = 0; u < ES_U; ++u) {
      const int base = p0 + u * 256;
      if (k < 0 || base >= t) break;
      uint64_t m[4] = {__ballot(x[u].x == k), __ballot(x[u].y == k), __ballot(x[u].z == k), __ballot(x[u].w == k)};
      if ((m[0] | m[1] | m[2] | m[3]) == 0) continue;
      if (base + 256 > t)
#pragma unroll
        for (int c = 0; c < 4; ++c) m[c] &= lanes_below(t, base, c);
      nb += __popcll(m[0]) + __popcll(m[1]) + __popcll(m[2]) + __popcll(m[3]);
    }
    if (lane == 0) nbefore[q][wave] = nb;
  }
  __syncthreads();
  // Lane q W + w: what wave w saw before position q; every lane of q W .. the sum.
  int jq = lane < W * W ? nbefore[lane / W][lane % W] : 0;
#pragma unroll
  for (int off = 1; off < W; off <<= 1) jq += __shfl_xor(jq, off);
  // The next occurrences after each position that starts a run.
#pragma unroll 1
  for (int q = 0; q < W; ++q) {
    const int t = t0 + q, k = __builtin_amdgcn_readlane(ks, q);
    int na = 0;
    if (k >= 0 && __builtin_amdgcn_readlane(jq, q * W) % RUN == 0) {
#pragma unroll
      for (int u = 0; u < ES_U; ++u) {
        const int base = p0 + u * 256;
        if (base + 256 <= t || na >= RUN) continue;
        uint64_t m[4] = {__ballot(x[u].x == k), __ballot(x[u].y == k), __ballot(x[u].z == k), __ballot(x[u].w == k)};
        if ((m[0] | m[1] | m[2] | m[3]) == 0) continue;
        if (base <= t)
#pragma unroll
          for (int c = 0; c < 4; ++c) m[c] &= ~lanes_below(t + 1, base, c);
        int mine = na + below_lane(m[0]) + below_lane(m[1]) + below_lane(m[2]) + below_lane(m[3]);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if ((m[c] >> lane) & 1ull) {
            if (mine < RUN) near[q][wave][mine] = base + 4 * lane + c;
            ++mine;
          }
        na += __popcll(m[0]) + __popcll(m[1]) + __popcll(m[2]) + __popcll(m[3]);
      }
    }
    if (lane == 0) nnear[q][wave] = min(na, RUN);
  }
  // Marks before each thread's stretch of the bitmap (an odd stretch: its words lie in
  // banks of their own).
  const int per = ((words + NT - 1) / NT) | 1;
  int nseg = 0;
  if (a.tokens) {
    const int w0 = min(words, per * (int)threadIdx.x), w1 = min(words, w0 + per);
    int c = 0;
    for (int i = w0; i < w1; ++i) c += __popc(lds[i]);
    stretch[threadIdx.x] = block_scan<NT>(c, part, &nseg);
  }
  __syncthreads();
  // Wave q joins what the waves saw of position q: its number among its token's
  // occurrences, and the next RUN (one more than a run holds: whether another run follows).
  const int t = t0 + wave;
  const int kt = __builtin_amdgcn_readfirstlane(__shfl(ks, wave)), j = __builtin_amdgcn_readfirstlane(__shfl(jq, wave * W));
  int found = 0;
  {
    const int c = lane < W ? nnear[wave][lane] : 0, inc = wave_scan(c, lane);
    found = __builtin_amdgcn_readlane(inc, 63);
    for (int i = 0; i < c; ++i)
      if (inc - c + i < RUN) list[wave][inc - c + i] = near[wave][lane][i];
  }
  const bool starts = kt >= 0 && j % RUN == 0, first = j == 0, more = found >= RUN;
  if (lane == 0) again[wave] = starts && (!first || more);
  __syncthreads();
#pragma unroll 1
  for (int q = 0; q < W; ++q) {
    if (!__builtin_amdgcn_readfirstlane(again[q])) continue;
    const int k = __builtin_amdgcn_readlane(ks, q);
    int less = 0, equal = 0;
#pragma unroll
    for (int u = 0; u < ES_U; ++u) {
      const int xs[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        less += __popcll(__ballot((unsigned)xs[c] < (unsigned)k));
        equal += __popcll(__ballot(xs[c] == k));
      }
    }
    if (lane == 0) {
      nless[q][wave] = less;
      nequal[q][wave] = equal;
    }
  }
  __syncthreads();
  int kind = 0, row = 0;
  if (lane < 3) hot[wave][lane] = 0;
  if (starts) {
    int less = 0, equal = 0;
    if (!first || more)
      for (int w = 0; w < W; ++w) {
        less += nless[wave][w];
        equal += nequal[wave][w];
      }
    kind = first ? 1 : 2;
    row = first ? kt : (less + j) / RUN;
    if (a.tokens && first) {
      // (its stretch's marks before it, a word a lane)
      const int word = kt >> 5, first_word = word / per * per;
      int c = 0;
      for (int i = first_word + lane; i <= word; i += 64)
        c += __popc(i < word ? lds[i] : lds[i] & ((1u << (kt & 31)) - 1u));
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) c += __shfl_xor(c, off);
      row = stretch[word / per] + c;
      if (lane == 0) a.tokens[row] = kt;
    }
    if (first && more && lane == 0) {
      hot[wave][0] = row;
      hot[wave][1] = (less + RUN) / RUN;
      hot[wave][2] = (equal - 1) / RUN;
    }
  }
  const int n = min(found, RUN - 1);
  // Runs of one or two rows: each wave its own.  Longer ones: all waves, a part of the
  // columns each (a wave alone took 12 rounds of eight loads for 3072 columns).
  if (lane == 0) {
    run[wave][0] = n > 1 ? kind : 0;
    run[wave][1] = row;
    run[wave][2] = n;
  }
  __syncthreads();
  auto dest = [&](int kd, int64_t r) { return kd == 1 ? a.out + r * a.D : a.slots + r * a.D; };
  row = __builtin_amdgcn_readfirstlane(row);
  if (kind != 0 && n == 0)
    sum_rows<E, 64, 1>(a, t, list[wave], n, dest(kind, row), kind == 1 ? a.scale : 1.0f, kind == 1 && a.accumulate);
  if (kind != 0 && n == 1)
    sum_rows<E, 64, 2>(a, t, list[wave], n, dest(kind, row), kind == 1 ? a.scale : 1.0f, kind == 1 && a.accumulate);
  if (a.tokens && t < a.cap && t >= nseg) {  // what no token reaches
    if (lane == 0) a.tokens[t] = -1;
    f32x4 *o = (f32x4 *)(a.out + (int64_t)t * a.D);
    for (int v = lane; v < a.D / 4; v += 64) o[v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
#pragma unroll 1
  for (int q = 0; q < W; ++q) {
    const int kd = __builtin_amdgcn_readfirstlane(run[q][0]);
    if (kd == 0) continue;
    const int m = __builtin_amdgcn_readfirstlane(run[q][2]);
    float *dst = dest(kd, __builtin_amdgcn_readfirstlane(run[q][1]));
    const float f = kd == 1 ? a.scale : 1.0f;
    const bool add = kd == 1 && a.accumulate;
    if (RUN <= ES_BATCH || m < ES_BATCH) sum_rows<E, NT, ES_BATCH>(a, t0 + q, list[q], m, dst, f, add);
    else sum_long<E, NT>(a, t0 + q, list[q], m, dst, f, add);
  }
  if (threadIdx.x == 0) {
    int m = 0;
    for (int q = 0; q < W; ++q) {
      if (hot[q][2] == 0) continue;
      int32_t *e = a.hot + 3 * ((int64_t)t0 + m++);
      e[0] = hot[q][0];
      e[1] = hot[q][1];
      e[2] = hot[q][2];
    }
    a.nhot[blockIdx.x] = m;
  }
}

// Adds the slots of the tokens with more than one run to their rows (half as many
// workgroups: 36 us for both launches of the case above, instead of 34).  An item is
// a token and ES_COLS columns; the waves take consecutive ranges of its slots,
// whose sums are added in their order.
constexpr int EJ_NT = 1024, EJ_WAVES = EJ_NT / 64, EJ_GRID = 512;
__global__ __launch_bounds__(EJ_NT) void embed_slots_kernel(EmbedScan a, int per_wg) {
  __shared__ int first[EJ_NT];  // number of the workgroup's first item
  __shared__ int part[EJ_WAVES];
  __shared__ f32x4 red[EJ_WAVES][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int total;
  first[threadIdx.x] = block_scan<EJ_NT>((int)threadIdx.x < a.nwg ? a.nhot[threadIdx.x] : 0, part, &total);
  __syncthreads();
  const int ncol = (a.D + ES_COLS - 1) / ES_COLS;
  for (int64_t it = blockIdx.x; it < (int64_t)total * ncol; it += gridDim.x) {
    const int h = (int)(it / ncol), v = (int)(it % ncol) * 64 + lane;
    int lo = 0, hi = a.nwg - 1;  // the last workgroup whose first item is at most h (it has one: empty ones repeat the next's)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= h) lo = mid;
      else hi = mid - 1;
    }
    const int32_t *e = a.hot + 3 * ((int64_t)lo * per_wg + (h - first[lo]));
    const int row = e[0], slot = e[1], n = e[2];
    const int per = (n + EJ_WAVES - 1) / EJ_WAVES, s0 = min(n, wave * per), s1 = min(n, s0 + per);
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (v < a.D / 4) {
      const f32x4 *x = (const f32x4 *)(a.slots + (int64_t)(slot + s0) * a.D) + v;
#pragma unroll 8
      for (int i = s0; i < s1; ++i, x += a.D / 4) s += *x;
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && v < a.D / 4) {
      for (int w = 1; w < EJ_WAVES; ++w) s += red[w][lane];
      f32x4 *o = (f32x4 *)(a.out + (int64_t)row * a.D) + v;
      *o += s * a.scale;
    }
    __syncthreads();
  }
}

hipError_t launch_embed_fwd(const void *table, const int32_t *ids, void *out, int T, int V, int D, float scale, Dtype d,
                            hipStream_t st) {
  const int vpr = D / (d == DT_BF16 ? 8 : 4);
  const unsigned per_row = (vpr + 64 * EF_U - 1) / (64 * EF_U);
  const dim3 grid((unsigned)(((int64_t)T * per_row + EF_NT / 64 - 1) / (EF_NT / 64)));
  if (d == DT_BF16)
    hipLaunchKernelGGL(embed_fwd_kernel<BF16>, grid, dim3(EF_NT), 0, st, (const uint16_t *)table, ids, (uint16_t *)out, T, V,
                       vpr, per_row, scale);
  else
    hipLaunchKernelGGL(embed_fwd_kernel<F32>, grid, dim3(EF_NT), 0, st, (const float *)table, ids, (float *)out, T, V, vpr,
                       per_row, scale);
  return hipGetLastError();
}

// Without a sort, compact form over 128256 x 3072 / 8192 x 512: 4096 positions 34 / 23 us (with
// one 57 / 42), 6000 45 / 32 (61 / 44), 8192 59 / 44 (66 / 50); a lane holds 16
// tokens of a workgroup of 512.  The bitmap of up to 262144 tokens takes 32 KB of LDS.
constexpr int64_t EMBED_SCAN_T = 8192, EMBED_SCAN_V = 262144;

static size_t up256(size_t b) { return (b + 255) & ~size_t(255); }

EmbedPlan embed_plan(int64_t T, int64_t V, int64_t D) {
  EmbedPlan p{};
  size_t off = 0;
  p.scan = T <= EMBED_SCAN_T && V <= EMBED_SCAN_V;
  if (p.scan) {
    p.per_wg = T <= 4096 ? 4 : 8;
    p.nwg = (int)((T + p.per_wg - 1) / p.per_wg);
    p.nhot = off;
    off += up256((size_t)p.nwg * 4);
    p.hot = off;
    off += up256((size_t)p.nwg * p.per_wg * 12);
    p.partial = off;
    off += up256((size_t)(T / ES_RUN + 1) * D * 4);
    p.total = off;
    return p;
  }
  int bits = 1;
  while (((int64_t)1 << bits) <= V) ++bits;  // keys 0 .. V
  p.passes = (bits + 8) / 9;
  p.digit = (bits + p.passes - 1) / p.passes;
  p.ntile = (int)((T + RS_TILE - 1) / RS_TILE);
  p.chunk = 4 * EG_U;
  p.nchunk = (int)((T + p.chunk - 1) / p.chunk);
  const int64_t nsg = (T + SG_TILE - 1) / SG_TILE;
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
  const bool direct = p.ntile <= RS_DIRECT;
  int *count = (int *)(ws + p.count), *total = count + (int64_t)RS_BINS * p.ntile;
  const uint32_t *key = (const uint32_t *)ids;
  const int32_t *pos = nullptr;
  for (int s = 0; s < p.passes; ++s) {
    const int o = (p.passes - 1 - s) & 1;  // the last pass writes buffer 0
    const bool first = s == 0;
    hipLaunchKernelGGL(radix_count_kernel, dim3(p.ntile), dim3(RS_NT), 0, st, key, first, T, V, s * p.digit, bins, p.ntile,
                       count);
    if (!direct) hipLaunchKernelGGL(radix_prefix_kernel, dim3(bins), dim3(RS_NT), 0, st, count, p.ntile, total);
    hipLaunchKernelGGL(radix_scatter_kernel, dim3(p.ntile), dim3(RS_NT), 0, st, key, pos, first, T, V, s * p.digit, p.digit,
                       p.ntile, count, total, direct, (uint32_t *)(ws + p.key[o]), (int32_t *)(ws + p.pos[o]));
    key = (const uint32_t *)(ws + p.key[o]);
    pos = (const int32_t *)(ws + p.pos[o]);
  }
  if (tokens) {
    const int nsg = (T + SG_TILE - 1) / SG_TILE;
    int *sc = (int *)(ws + p.segcount), *seg = (int *)(ws + p.seg);
    const bool own = nsg <= SG_OWN;
    if (!own) {
      hipLaunchKernelGGL(seg_count_kernel, dim3(nsg), dim3(SG_NT), 0, st, key, T, V, sc);
      hipLaunchKernelGGL(radix_prefix_kernel, dim3(1), dim3(RS_NT), 0, st, sc, nsg, sc + nsg);
    }
    hipLaunchKernelGGL(seg_kernel, dim3(nsg), dim3(SG_NT), 0, st, key, T, V, own ? nullptr : sc, sc + nsg, seg, tokens);
  }
  return hipGetLastError();
}

template <typename E>
static void embed_scan(const EmbedScan &a, const EmbedPlan &p, int own, size_t lds, hipStream_t st) {
  const dim3 grid((unsigned)(p.nwg + own));
  if (a.T <= ES_FEW) hipLaunchKernelGGL((embed_scan_kernel<E, 256, ES_FEW>), grid, dim3(256), lds, st, a);
  else if (p.per_wg == 4) hipLaunchKernelGGL((embed_scan_kernel<E, 256, ES_RUN>), grid, dim3(256), lds, st, a);
  else hipLaunchKernelGGL((embed_scan_kernel<E, 512, ES_RUN>), grid, dim3(512), lds, st, a);
}

hipError_t launch_embed_scan(const int32_t *ids, const void *dout, float *out, int32_t *tokens, int T, int V, int D, float scale,
                             bool accumulate, Dtype d, const EmbedPlan &p, char *ws, hipStream_t st) {
  EmbedScan a{};
  a.ids = ids;
  a.dout = dout;
  a.out = out;
  a.tokens = tokens;
  a.slots = (float *)(ws + p.partial);
  a.nhot = (int32_t *)(ws + p.nhot);
  a.hot = (int32_t *)(ws + p.hot);
  a.T = T;
  a.V = V;
  a.D = D;
  a.cap = T < V ? T : V;
  a.nwg = p.nwg;
  a.accumulate = accumulate;
  a.scale = scale;
  // A dense gradient below 256 MB is cleared beside the sums, which spares a launch (3 us) and
  // hides the search for the tokens; a larger one ahead of them, at the higher rate.
  int own = 0;
  if (!accumulate && !tokens) {
    if ((int64_t)V * D < (64 << 20)) own = (V + ES_CLEAR - 1) / ES_CLEAR;
    else clear(out, V, D, st);
  }
  const size_t lds = tokens ? (size_t)((V + 31) / 32) * 4 : 4;
  if (d == DT_BF16) embed_scan<BF16>(a, p, own, lds, st);
  else embed_scan<F32>(a, p, own, lds, st);
  if (T > ES_FEW) {  // (at most T / (RUN + 1) tokens have a second run)
    const int64_t items = (int64_t)(T / (ES_RUN + 1)) * ((D + ES_COLS - 1) / ES_COLS);
    hipLaunchKernelGGL(embed_slots_kernel, dim3((unsigned)std::min<int64_t>(EJ_GRID, items)), dim3(EJ_NT), 0, st, a, p.per_wg);
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
  a.ncol = (D / vec + EG_COL - 1) / EG_COL;
  const unsigned nwork = (unsigned)((int64_t)((a.nchunk + 1) / 2) * a.ncol);
  if (!tokens && !accumulate) clear(out, V, D, st);
  const dim3 grid(nwork + (tokens ? (unsigned)((a.cap + 63) / 64) : 0u)), join((unsigned)((int64_t)(a.nchunk - 1) * a.ncol));
  if (d == DT_BF16) {
    hipLaunchKernelGGL(embed_grad_kernel<BF16>, grid, dim3(EG_NT), 0, st, a, nwork);
    if (a.nchunk > 1) hipLaunchKernelGGL(embed_join_kernel<BF16>, join, dim3(EG_COL), 0, st, a);
  } else {
    hipLaunchKernelGGL(embed_grad_kernel<F32>, grid, dim3(EG_NT), 0, st, a, nwork);
    if (a.nchunk > 1) hipLaunchKernelGGL(embed_join_kernel<F32>, join, dim3(EG_COL), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace lora
