// x8prod.hip -- the rank-r products of the LoRA backward whose input x is kept in
// 8 bits (act8.hpp): u = x A^T where it is not saved, and the token reductions
//   dA = du^T x,  dB = s dy^T u.
// Codes are whole numbers up to 127, exact in bf16, so a product on the matrix
// cores takes them as they are; a scale belongs to a row and 128 columns of x and goes
// to the other side of the product: in u to the group's sum, in dA to du.  du and u
// are fp32 and stay so: v as the sum of three bf16, which hold its 24 bits.  (Two leave
// 2^-18 of it, 2e-6 of the gradient's norm; one 2^-9.  The third product takes 1 us of
// the 22 of 8192 -> 3072 at 4096 tokens.)
#include <algorithm>

#include "act8.hpp"
#include "launch.hpp"

namespace lora {

// 8 codes as a matrix-core operand of bf16 (whole numbers up to 127: no rounding).
__device__ __forceinline__ u32x4 x8_operand(uint2 q) {
  float f[8];
  act8_floats(q, f);
  u32x4 r;
#pragma unroll
  for (int d = 0; d < 4; ++d) r[d] = pack_bf16x2(f[2 * d], f[2 * d + 1]);
  return r;
}

// ---- u = x A^T -----------------------------------------------------------------------
// A workgroup of 8 waves takes 16 MB tokens and a range of groups; each wave every
// eighth group, all ranks.  Lane (row or rank l % 16, quarter l / 16) holds 32
// consecutive columns of a group: the four products of a group take them 8 at a
// time, in the same order on both sides.
constexpr int X8D_NW = 8;

template <int JB, int MB>
__global__ __launch_bounds__(64 * X8D_NW) void x8_down_kernel(X8Down a, int groups_per) {
  __shared__ float red[X8D_NW / 2][16 * MB][JB * 16 + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q4 = lane >> 4;
  const int ng = (a.K + ACT8_G - 1) / ACT8_G;
  const int g1 = min(ng, ((int)blockIdx.y + 1) * groups_per);
  const int t0 = blockIdx.x * 16 * MB;
  f32x4 tot[MB][JB];
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int j = 0; j < JB; ++j) tot[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int g = blockIdx.y * groups_per + wave; g < g1; g += X8D_NW) {
    const int col = g * ACT8_G + q4 * 32;
    uint2 x[MB][4];
    u32x4 w[JB][4];
    float s[MB][4];
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      const int t = t0 + 16 * m + c;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[m][k] = make_uint2(0u, 0u);
        if (t < a.T && col + 8 * k < a.K) x[m][k] = *(const uint2 *)(a.x.codes + (int64_t)t * a.K + col + 8 * k);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ts = t0 + 16 * m + 4 * q4 + i;
        s[m][i] = ts < a.T ? a.x.scale[(int64_t)ts * ng + g] : 0.0f;
      }
    }
#pragma unroll
    for (int j = 0; j < JB; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[j][k] = j * 16 + c < a.r && col + 8 * k < a.K
                      ? ld16((const uint16_t *)a.A + (int64_t)(j * 16 + c) * a.K + col + 8 * k)
                      : zero16();
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      u32x4 xb[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) xb[k] = x8_operand(x[m][k]);
#pragma unroll
      for (int j = 0; j < JB; ++j) {
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) mma16(BF16(), acc, xb[k], w[j][k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) tot[m][j][i] = __builtin_fmaf(s[m][i], acc[i], tot[m][j][i]);
      }
    }
  }
  // the waves' sums, pairwise: element i of lane is token 4 q4 + i, rank 16 j + c
#pragma unroll
  for (int h = X8D_NW / 2; h >= 1; h /= 2) {
    __syncthreads();
    if (wave >= h && wave < 2 * h) {
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int j = 0; j < JB; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) red[wave - h][16 * m + 4 * q4 + i][16 * j + c] = tot[m][j][i];
    }
    __syncthreads();
    if (wave < h) {
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int j = 0; j < JB; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) tot[m][j][i] += red[wave][16 * m + 4 * q4 + i][16 * j + c];
    }
  }
  if (wave != 0) return;
  float *u = a.u + (int64_t)blockIdx.y * a.T * a.r;
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int j = 0; j < JB; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t0 + 16 * m + 4 * q4 + i, k = 16 * j + c;
        if (t < a.T && k < a.r) u[(int64_t)t * a.r + k] = tot[m][j][i];
      }
}

struct X8DownSplit {
  int mb, parts, groups;
};
static X8DownSplit x8_down_split(int64_t T, int64_t K) {
  const int64_t ng = (K + ACT8_G - 1) / ACT8_G;
  const int mb = T >= 1024 ? 2 : 1;
  const int64_t blocks = (T + 16 * mb - 1) / (16 * mb);
  // as many ranges as give each CU a workgroup, each of a group a wave at least
  const int64_t p = std::max<int64_t>(1, std::min<int64_t>({4, 256 / blocks, ng / X8D_NW}));
  const int64_t groups = (ng + p - 1) / p;
  return {mb, (int)((ng + groups - 1) / groups), (int)groups};
}
int x8_down_parts(int64_t T, int64_t K) { return x8_down_split(T, K).parts; }

template <int JB>
static hipError_t x8_down_jb(const X8Down &a, hipStream_t st) {
  const X8DownSplit s = x8_down_split(a.T, a.K);
  const dim3 grid((a.T + 16 * s.mb - 1) / (16 * s.mb), s.parts), block(64 * X8D_NW);
  if (s.mb == 1) hipLaunchKernelGGL((x8_down_kernel<JB, 1>), grid, block, 0, st, a, s.groups);
  else hipLaunchKernelGGL((x8_down_kernel<JB, 2>), grid, block, 0, st, a, s.groups);
  return hipGetLastError();
}
hipError_t launch_x8_down(const X8Down &a, hipStream_t st) {
  switch ((a.r + 15) / 16) {
    case 1: return x8_down_jb<1>(a, st);
    case 2: return x8_down_jb<2>(a, st);
    case 3:
    case 4: return x8_down_jb<4>(a, st);
    case 5:
    case 6:
    case 7:
    case 8: return x8_down_jb<8>(a, st);
  }
  return hipErrorInvalidValue;
}

// ---- dA = du^T x, dB = s dy^T u ------------------------------------------------------
// An item is 128 columns of x (a group: one scale a token) or of dy by 16 JB ranks,
// over a range of tokens.  Its waves take steps of 32 tokens in turn: lane (c = l % 16, g = l / 16)
// loads 8 columns of tokens 8 g .. 8 g + 7, and the 8 tokens of one of its columns are
// an operand whose reduction axis is the token axis; product q takes column 8 c + q of
// every c.  The waves' tiles are summed pairwise.
constexpr int X8P_NW = 8, X8P_ROWS = 32;

struct X8Unit {
  const void *X;
  const float *scale, *V;
  float *out;
  int L, ng, vparts, t0, t1, cb, jg;
  float mult;
  bool transposed;  // out [r][L], else [L][r]
};

template <int JB, bool X8>
__device__ __forceinline__ void x8_item(const X8Prod &a, const X8Unit &n, float (*red)[ACT8_G][JB * 16 + 1]) {
  constexpr uint32_t OOB = 0x80000000u;
  constexpr int ES = X8 ? 1 : 2, XW = X8 ? 2 : 4;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = n.cb * ACT8_G + 8 * c, r = a.r;
  const int64_t plane = (int64_t)a.T * r;
  struct Step {
    uint32_t x[8][XW];
    float v[JB][8], s[8];
  };
  // Loads go through buffer resources based at the step's first token: tokens past the range,
  // columns past L and ranks past r read zeros.
  auto load = [&](int tb, Step &st) {
    const int rows = max(0, min(X8P_ROWS, n.t1 - tb));
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
        (void *)((const char *)n.X + (int64_t)tb * n.L * ES), (short)0, rows * n.L * ES, 0x00020000);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t off = col < n.L ? (uint32_t)(((8 * g + i) * n.L + col) * ES) : OOB;
      if constexpr (X8) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 t = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rx, off, 0, 0));
        st.x[i][0] = t[0];
        st.x[i][1] = t[1];
      } else {
        const u32x4 t = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, off, 0, 0));
#pragma unroll
        for (int k = 0; k < 4; ++k) st.x[i][k] = t[k];
      }
    }
    if constexpr (X8) {
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
          (void *)(n.scale + (int64_t)tb * n.ng), (short)0, rows * n.ng * 4, 0x00020000);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        st.s[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, ((8 * g + i) * n.ng + n.cb) * 4, 0, 0));
    }
    for (int p = 0; p < n.vparts; ++p) {
      const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(
          (void *)(n.V + p * plane + (int64_t)tb * r), (short)0, rows * r * 4, 0x00020000);
#pragma unroll
      for (int j = 0; j < JB; ++j) {
        const int k = n.jg + 16 * j + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t off = k < r ? (uint32_t)(((8 * g + i) * r + k) * 4) : OOB;
          const float v = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rv, off, 0, 0));
          st.v[j][i] = p == 0 ? v : st.v[j][i] + v;
        }
      }
    }
  };
  f32x4 acc[8][JB];
#pragma unroll
  for (int q = 0; q < 8; ++q)
#pragma unroll
    for (int j = 0; j < JB; ++j) acc[q][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto compute = [&](const Step &st) {
    u32x4 vb[JB][3], xt[8];
#pragma unroll
    for (int j = 0; j < JB; ++j) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = X8 ? st.v[j][i] * st.s[i] : st.v[j][i];
#pragma unroll
      for (int p = 0; p < 3; ++p) {  // each the next bits of what is left
#pragma unroll
        for (int d = 0; d < 4; ++d) vb[j][p][d] = pack_bf16x2(v[2 * d], v[2 * d + 1]);
        if (p == 2) break;
        float h[8];
        unpack_vec(BF16(), vb[j][p], h);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] -= h[i];
      }
    }
    if constexpr (X8) {
      // column q of the 8 tokens: byte q of each
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)(int8_t)(st.x[i][q >> 2] >> (8 * (q & 3)));
#pragma unroll
        for (int d = 0; d < 4; ++d) xt[q][d] = pack_bf16x2(f[2 * d], f[2 * d + 1]);
      }
    } else {
      u32x4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = u32x4{st.x[i][0], st.x[i][1], st.x[i][2], st.x[i][3]};
      transpose_block(BF16(), x, xt);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q)
#pragma unroll
      for (int j = 0; j < JB; ++j) {
#pragma unroll
        for (int p = 0; p < 3; ++p) mma16(BF16(), acc[q][j], xt[q], vb[j][p]);
      }
  };
  {
    Step cur, nxt;
    int tb = n.t0 + wave * X8P_ROWS;
    if (tb < n.t1) load(tb, cur);
    for (; tb < n.t1; tb += X8P_NW * X8P_ROWS) {
      load(min(tb + X8P_NW * X8P_ROWS, n.t1), nxt);  // (at the end: an empty resource)
      compute(cur);
      cur = nxt;
    }
  }
  // acc[q][j] element i: column (4 g + i) 8 + q, rank 16 j + c
#pragma unroll
  for (int h = X8P_NW / 2; h >= 1; h /= 2) {
    __syncthreads();
    if (wave >= h && wave < 2 * h) {
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int j = 0; j < JB; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) red[wave - h][(4 * g + i) * 8 + q][16 * j + c] = acc[q][j][i];
    }
    __syncthreads();
    if (wave < h) {
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int j = 0; j < JB; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[q][j][i] += red[wave][(4 * g + i) * 8 + q][16 * j + c];
    }
  }
  // the tile to LDS, and from there out in whole rows
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
#pragma unroll
      for (int j = 0; j < JB; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[0][(4 * g + i) * 8 + q][16 * j + c] = n.mult * acc[q][j][i];
  }
  __syncthreads();
  const int cols = min(ACT8_G, n.L - n.cb * ACT8_G), ranks = min(16 * JB, r - n.jg);
  for (int i = threadIdx.x; i < ACT8_G * JB * 16; i += 64 * X8P_NW) {
    if (n.transposed) {
      const int k = i / ACT8_G, l = i % ACT8_G;
      if (k < ranks && l < cols) n.out[(int64_t)(n.jg + k) * n.L + n.cb * ACT8_G + l] = red[0][l][k];
    } else {
      const int l = i / (JB * 16), k = i % (JB * 16);
      if (k < ranks && l < cols) n.out[(int64_t)(n.cb * ACT8_G + l) * r + n.jg + k] = red[0][l][k];
    }
  }
}

// Workgroups: the items of dB (twice the bytes an item), then those of dA, each in
// `parts` ranges of tokens, which write to their own planes where there are several.
template <int JB>
__global__ __launch_bounds__(64 * X8P_NW) void x8_prod_kernel(X8Prod a, int parts, int chunk, int items_b) {
  __shared__ float red[X8P_NW / 2][ACT8_G][JB * 16 + 1];
  const int nz = (a.r + 16 * JB - 1) / (16 * JB);
  const int unit = blockIdx.x, part = unit % parts;
  int item = unit / parts;
  const bool dB = item < items_b;
  if (!dB) item -= items_b;
  const int64_t ra = (int64_t)a.r * a.K, rb = (int64_t)a.r * a.N;
  float *const plane = parts > 1 ? a.planes + part * (ra + rb) : nullptr;
  X8Unit n;
  n.cb = item / nz;
  n.jg = item % nz * 16 * JB;
  n.t0 = part * chunk;
  n.t1 = min(a.T, n.t0 + chunk);
  n.X = dB ? a.dy : (const void *)a.x.codes;
  n.scale = a.x.scale;
  n.V = dB ? a.u : a.du;
  n.vparts = dB ? a.u_parts : a.du_parts;
  n.L = dB ? a.N : a.K;
  n.ng = (a.K + ACT8_G - 1) / ACT8_G;
  n.mult = dB ? a.scale : 1.0f;
  n.transposed = !dB;
  n.out = dB ? (plane ? plane + ra : a.dB) : (plane ? plane : a.dA);
  if (dB) x8_item<JB, false>(a, n, red);
  else x8_item<JB, true>(a, n, red);
}

// dA and dB as the sums of the planes, in ascending order.
__global__ __launch_bounds__(256) void x8_sum_kernel(const float *planes, int np, int64_t na, int64_t n, float *dA, float *dB) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;  // (na and n are multiples of 8)
  if (i >= n) return;
  f32x4 s = *(const f32x4 *)(planes + i);
  for (int p = 1; p < np; ++p) s += *(const f32x4 *)(planes + p * n + i);
  *(f32x4 *)(i < na ? dA + i : dB + (i - na)) = s;
}

static int64_t x8_items(int64_t L, int64_t r) { return (L + ACT8_G - 1) / ACT8_G * ((r + (r <= 16 ? 15 : 31)) / (r <= 16 ? 16 : 32)); }

X8Plan x8_plan(int64_t T, int64_t K, int64_t N, int64_t r) {
  constexpr int64_t STEP = X8P_NW * X8P_ROWS;
  const int64_t items = x8_items(K, r) + x8_items(N, r);
  // two workgroups a CU, each of a step of every wave at least
  const int64_t p = std::max<int64_t>(1, std::min<int64_t>({16, 512 / items, T / STEP}));
  const int64_t chunk = ((T + p - 1) / p + STEP - 1) / STEP * STEP;
  const int64_t parts = (T + chunk - 1) / chunk;
  return {(int)parts, (int)chunk, parts > 1 ? (size_t)(parts * r * (K + N) * 4) : 0};
}

hipError_t launch_x8_prod(const X8Prod &a, hipStream_t st) {
  const X8Plan p = x8_plan(a.T, a.K, a.N, a.r);
  const int items_b = (int)x8_items(a.N, a.r), items = items_b + (int)x8_items(a.K, a.r);
  const dim3 grid(items * p.parts), block(64 * X8P_NW);
  if (a.r <= 16) hipLaunchKernelGGL((x8_prod_kernel<1>), grid, block, 0, st, a, p.parts, p.chunk, items_b);
  else hipLaunchKernelGGL((x8_prod_kernel<2>), grid, block, 0, st, a, p.parts, p.chunk, items_b);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  const int64_t na = (int64_t)a.r * a.K, n = na + (int64_t)a.r * a.N;
  hipLaunchKernelGGL(x8_sum_kernel, dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, st, a.planes, p.parts, na, n, a.dA, a.dB);
  return hipGetLastError();
}

}  // namespace lora
